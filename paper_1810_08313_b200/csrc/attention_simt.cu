// Attention over packed sequences and its gradient on the CUDA cores: fp32 tensors, and the bf16 ones that the tensor-core
// kernels do not take (see attention.cuh for the formulas and attention_tc.cu for the others).  The entry points are here, too.
//
// One CTA of 256 threads per tile of 64 rows of one head, or of 128 threads per 32 rows where those are too few for the SMs; blocks
// of 64 keys pass through shared memory once each, and scores never leave the SM.  (Heads of more than 128: 256 threads, 32 rows and 32
// keys.)  Thread (ty, tx), 16 to a row of threads, has the rows ty R .. + R - 1 and the keys tx + 16 c of a block of scores; the
// loads of a block are requested together; operands are read four elements of a head at a time, rows padded by four floats, so that the reads of a quarter warp fall into distinct banks and 4 x 4 x 4 multiply-adds
// need 8 reads of 16 bytes.  The second products read the scores back from shared memory the same way.  Forward: a running
// maximum and sum a row.  Backward: one launch with CTAs for dk and dv, tiles of keys which take all the queries of their group's
// heads, and others for dq, tiles of queries: the scores are formed twice, and no sum depends on an order of arrival.  Where
// there are few tiles of keys, a cluster of CTAs shares the queries of a tile, and its first one adds up the parts, in order, out
// of the others' shared memory.
// Bound by the reads of shared memory that feed the multiply-adds, and with few rows by the chain of blocks of the longest sequence:
// fp32, 4096 rows of 8 heads of 128 on 2 in three sequences: 468 us forward (28 TFLOP/s of what is visible), 1488 us backward; 2 x
// 513 rows of 6 heads of 64 on 2 in five: 27 and 51 us.
#include "attention.cuh"

namespace ls {
namespace attn {
namespace {

// HD: head_dim at most; RB: rows of a tile
template <int HD, int RB>
struct Way {
  static constexpr int NT = RB == 32 && HD <= 128 ? 128 : 256;       // threads
  static constexpr int B = RB, R = RB * 16 / NT;  // rows of a tile, of a thread
  static constexpr int K = HD > 128 ? 2 : 4;      // keys of a thread
  static constexpr int N = 16 * K;                // of a block
  static constexpr int P = HD + 4;                // floats between rows of an operand
  static constexpr int PS = N + 4;                // of the scores
  static constexpr int C = HD / 16;               // result columns of a thread: 4 tx + 64 c .. + 3, or tx + 16 c below 64
  static constexpr int rows = B * P, block = N * P, scores = B * PS;
};

__device__ __forceinline__ float4 four(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 four(const __nv_bfloat16* p) {
  const uint2 t = *reinterpret_cast<const uint2*>(p);
  return make_float4(__uint_as_float(t.x << 16), __uint_as_float(t.x & 0xFFFF0000u), __uint_as_float(t.y << 16),
                     __uint_as_float(t.y & 0xFFFF0000u));
}
// rows [r0, r0 + ROWS) of a head into shared memory as floats; zeros outside the tensor and the head.  quads: rows are whole fours of
// elements that start on their boundary
template <typename T, typename W, int HD, int ROWS>
__device__ __forceinline__ void load_tile(float* dst, const T* src, int64_t row, int64_t r0, int64_t rows, int hd, bool quads) {
  constexpr int P = HD + 4;
  if (quads) {
    constexpr int Q = HD / 4, N = ROWS * Q / W::NT;
    static_assert(ROWS * Q % W::NT == 0, "whole rounds");
    float4 v[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int i = n * W::NT + threadIdx.x, r = i / Q, c = (i - r * Q) * 4;
      v[n] = r0 + r < rows && c < hd ? four(src + (r0 + r) * row + c) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int i = n * W::NT + threadIdx.x, r = i / Q, c = (i - r * Q) * 4;
      *reinterpret_cast<float4*>(dst + r * P + c) = v[n];
    }
    return;
  }
  for (int i = threadIdx.x; i < ROWS * HD; i += W::NT) {
    const int r = i / HD, c = i - r * HD;
    dst[r * P + c] = r0 + r < rows && c < hd ? to_f32(src[(r0 + r) * row + c]) : 0.f;
  }
}

// two tiles at once, so that all their loads are on their way together
template <typename T, typename W, int HD, int ROWS>
__device__ __forceinline__ void load_two(float* d1, const T* s1, int64_t row1, float* d2, const T* s2, int64_t row2, int64_t r0, int64_t rows,
                                         int hd, bool quads) {
  if (!quads) {
    load_tile<T, W, HD, ROWS>(d1, s1, row1, r0, rows, hd, false);
    load_tile<T, W, HD, ROWS>(d2, s2, row2, r0, rows, hd, false);
    return;
  }
  constexpr int P = HD + 4, Q = HD / 4, N = ROWS * Q / W::NT;
  float4 v[N], w[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int i = n * W::NT + threadIdx.x, r = i / Q, c = (i - r * Q) * 4;
    const bool in = r0 + r < rows && c < hd;
    v[n] = in ? four(s1 + (r0 + r) * row1 + c) : make_float4(0.f, 0.f, 0.f, 0.f);
    w[n] = in ? four(s2 + (r0 + r) * row2 + c) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int i = n * W::NT + threadIdx.x, r = i / Q, c = (i - r * Q) * 4;
    *reinterpret_cast<float4*>(d1 + r * P + c) = v[n];
    *reinterpret_cast<float4*>(d2 + r * P + c) = w[n];
  }
}

// s[r][c] = x row (ty R + r) . y row (tx + 16 c)
template <typename W, int HD>
__device__ __forceinline__ void dots(const float* x, const float* y, int ty, int tx, float (&s)[W::R][W::K]) {
#pragma unroll
  for (int r = 0; r < W::R; ++r)
#pragma unroll
    for (int c = 0; c < W::K; ++c) s[r][c] = 0.f;
#pragma unroll 4
  for (int d = 0; d < HD; d += 4) {
    float4 a[W::R], b[W::K];
#pragma unroll
    for (int r = 0; r < W::R; ++r) a[r] = *reinterpret_cast<const float4*>(x + (ty * W::R + r) * W::P + d);
#pragma unroll
    for (int c = 0; c < W::K; ++c) b[c] = *reinterpret_cast<const float4*>(y + (tx + 16 * c) * W::P + d);
#pragma unroll
    for (int r = 0; r < W::R; ++r)
#pragma unroll
      for (int c = 0; c < W::K; ++c)
        s[r][c] = fmaf(a[r].w, b[c].w, fmaf(a[r].z, b[c].z, fmaf(a[r].y, b[c].y, fmaf(a[r].x, b[c].x, s[r][c]))));
  }
}

// the column of a head that is c-th of thread tx
template <int HD>
__device__ __forceinline__ int column(int tx, int c) {
  return HD >= 64 ? (c & ~3) * 16 + tx * 4 + (c & 3) : tx + 16 * c;
}
// acc[r][c] += sum over j of s[ty R + r][j] y[j][column c]
template <typename W, int HD>
__device__ __forceinline__ void accumulate(const float* s, const float* y, int ty, int tx, float (&acc)[W::R][W::C]) {
#pragma unroll 2
  for (int j = 0; j < W::N; j += 4) {
    float4 a[W::R];
#pragma unroll
    for (int r = 0; r < W::R; ++r) a[r] = *reinterpret_cast<const float4*>(s + (ty * W::R + r) * W::PS + j);
#pragma unroll
    for (int jj = 0; jj < 4; ++jj) {
      float b[W::C];
      const float* row = y + (j + jj) * W::P;
      if constexpr (HD >= 64) {
#pragma unroll
        for (int c = 0; c < W::C; c += 4) {
          const float4 t = *reinterpret_cast<const float4*>(row + column<HD>(tx, c));
          b[c] = t.x; b[c + 1] = t.y; b[c + 2] = t.z; b[c + 3] = t.w;
        }
      } else {
#pragma unroll
        for (int c = 0; c < W::C; ++c) b[c] = row[column<HD>(tx, c)];
      }
#pragma unroll
      for (int r = 0; r < W::R; ++r) {
        const float f = jj == 0 ? a[r].x : jj == 1 ? a[r].y : jj == 2 ? a[r].z : a[r].w;
#pragma unroll
        for (int c = 0; c < W::C; ++c) acc[r][c] = fmaf(f, b[c], acc[r][c]);
      }
    }
  }
}

// Writes acc[r][c] * by[r] to the rows r0 + ty R + r of the tensor; returns whether all of the thread's numbers are finite.
template <typename T, typename W, int HD>
__device__ __forceinline__ bool write_rows(T* dst, int64_t row, int64_t r0, int64_t rows, int hd, int ty, int tx,
                                           const float (&acc)[W::R][W::C], const float (&by)[W::R], uint32_t* bad) {
  bool good = true;
#pragma unroll
  for (int r = 0; r < W::R; ++r) {
    const int64_t i = r0 + ty * W::R + r;
    if (i >= rows) continue;
    bool fine = true;
#pragma unroll
    for (int c = 0; c < W::C; ++c) {
      const int d = column<HD>(tx, c);
      const float x = acc[r][c] * by[r];
      fine = fine && fabsf(x) < INFINITY;
      if (d < hd) dst[i * row + d] = from_f32<T>(x);
    }
    if (!fine) bad[ty * W::R + r] = 1u;
    good = good && fine;
  }
  return good;
}

// The tile's rows that are not finite, shared out over the warps: this warp's, from row first_bad() on.
template <typename W>
__device__ __forceinline__ int first_bad() { return (threadIdx.x >> 5) * (W::B * 32 / W::NT); }
template <typename W>
__device__ __forceinline__ uint32_t bad_rows(const uint32_t* bad) {
  constexpr int N = W::B * 32 / W::NT;
  static_assert(N <= 32, "bits of a word");
  const int lane = threadIdx.x & 31;
  return __ballot_sync(0xffffffffu, lane < N && bad[first_bad<W>() + lane % N] != 0u);
}

// sum or maximum over the 16 threads of a row
__device__ __forceinline__ float row_total(float x) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}
__device__ __forceinline__ float row_max(float x) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) x = max_nan(x, __shfl_xor_sync(0xffffffffu, x, o));
  return x;
}

// CTAs of an SM that registers have to leave room for: with heads of up to 32 the rare ways (forward_rows and the others) would take more
// than the tiles do.  (0: as the compiler sees fit.)
template <int HD, int RB>
constexpr int least_ctas(bool grad) { return HD > 32 ? 0 : RB == 64 ? 2 : grad ? 3 : 5; }

template <typename T, int HD, int RB>
__global__ void __launch_bounds__(Way<HD, RB>::NT, least_ctas<HD, RB>(false))
attention_kernel(const __grid_constant__ Args a, const bool quads) {
  using W = Way<HD, RB>;
  extern __shared__ __align__(16) float sm[];
  float* sq = sm;
  float* sk = sq + W::rows;
  float* sv = sk + W::block;
  float* sp = sv + W::block;
  __shared__ uint32_t bad[W::B];
  __shared__ int start[W::B];
  const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15, hd = a.head_dim;
  grid_dep_wait();
  grid_dep_launch();
  // the rows with the most keys first
  const int tiles = (int)((a.tokens + W::B - 1) / W::B);
  const int head = blockIdx.x % a.heads, rest = blockIdx.x / a.heads, rep = rest % a.m;
  const int64_t r0 = (int64_t)(tiles - 1 - rest / a.m) * W::B;
  const int kvh = head / (a.heads / a.kv_heads);
  load_tile<T, W, HD, W::B>(sq, head_ptr<const T>(a.q, rep, head, hd), a.q.row, r0, a.tokens, hd, quads);
  const Bounds bounds(a, rep);
  if (tid < W::B) {                        // (whole warps)
    int end;
    bad[tid] = 0u;
    bounds.rows((int)r0 + (tid & ~31), &start[tid], &end);
  }
  __syncthreads();
  const float scale2 = a.scale * kLog2e;
  float acc[W::R][W::C] = {}, top[W::R], sum[W::R];
#pragma unroll
  for (int r = 0; r < W::R; ++r) { top[r] = -INFINITY; sum[r] = 0.f; }
  const int64_t end = min(r0 + W::B, a.tokens);
  for (int64_t j0 = bounds.first_key((int)r0); j0 < end; j0 += W::N) {
    load_two<T, W, HD, W::N>(sk, head_ptr<const T>(a.k, rep, kvh, hd), a.k.row, sv, head_ptr<const T>(a.v, rep, kvh, hd), a.v.row, j0, a.tokens,
                             hd, quads);
    __syncthreads();
    float s[W::R][W::K];
    dots<W, HD>(sq, sk, ty, tx, s);
#pragma unroll
    for (int r = 0; r < W::R; ++r) {
      const int row = ty * W::R + r;
      float most = -INFINITY;
#pragma unroll
      for (int c = 0; c < W::K; ++c) {
        const int64_t j = j0 + tx + 16 * c;
        s[r][c] = j >= start[row] && j <= r0 + row ? s[r][c] * scale2 : -INFINITY;
        most = max_nan(most, s[r][c]);
      }
      most = max_nan(row_max(most), top[r]);
      const float ref = most == -INFINITY ? 0.f : most;
      const float keep = exp2f(top[r] - ref);
      top[r] = most;
      float part = 0.f;
#pragma unroll
      for (int c = 0; c < W::K; ++c) {
        const float p = exp2f(s[r][c] - ref);
        part += p;
        sp[row * W::PS + tx + 16 * c] = p;
      }
      sum[r] = fmaf(sum[r], keep, part);
#pragma unroll
      for (int c = 0; c < W::C; ++c) acc[r][c] *= keep;
    }
    __syncthreads();
    accumulate<W, HD>(sp, sv, ty, tx, acc);
    __syncthreads();
  }
  float by[W::R];
#pragma unroll
  for (int r = 0; r < W::R; ++r) {
    const int64_t i = r0 + ty * W::R + r;
    sum[r] = row_total(sum[r]);
    const bool none = start[ty * W::R + r] > i;
    if (none) {
#pragma unroll
      for (int c = 0; c < W::C; ++c) acc[r][c] = 0.f;
    }
    // (scores with a NaN or +inf, or of -inf only, have no softmax)
    const bool has = fabsf(top[r]) < INFINITY;
    by[r] = none ? 0.f : has ? 1.f / sum[r] : NAN;
    if (tx == 0 && i < a.tokens)
      a.lse[((int64_t)rep * a.heads + head) * a.tokens + i] = none ? 0.f : has ? fmaf(top[r], kLn2, logf(sum[r])) : top[r];
  }
  const bool good = write_rows<T, W, HD>(head_ptr<T>(a.out, rep, head, hd), a.out.row, r0, a.tokens, hd, ty, tx, acc, by, bad);
  if (__syncthreads_and(good)) return;
  const uint32_t ill = bad_rows<W>(bad);
  if (ill != 0u) forward_rows<T, HD / 32>(a, rep, head, (int)r0 + first_bad<W>(), ill);
}

// dot[r] = dout . out of the tile's rows: neighbouring threads share a row; out is loaded before, dout taken from shared memory
template <typename T, typename W, int HD, int ROWS>
struct RowDots {
  static constexpr int N = W::NT / ROWS, M = HD / 4 / N, P = HD + 4;
  float4 o[M];
  const T* row;
  __device__ __forceinline__ void fetch(const T* out, int64_t step, int64_t r0, int64_t rows, int hd, bool quads) {
    const int64_t i = r0 + threadIdx.x / N;
    row = i < rows ? out + i * step : nullptr;
    if (!quads) return;
#pragma unroll
    for (int n = 0; n < M; ++n) {
      const int e = (n * N + threadIdx.x % N) * 4;
      o[n] = row != nullptr && e < hd ? four(row + e) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
  }
  __device__ __forceinline__ void finish(float* dot, const float* sg, int hd, bool quads) const {
    const int r = threadIdx.x / N, part = threadIdx.x % N;
    float d = 0.f;
    if (quads) {
#pragma unroll
      for (int n = 0; n < M; ++n) {        // (dout is zeros behind the tensor and the head)
        const float4 g = *reinterpret_cast<const float4*>(sg + r * P + (n * N + part) * 4);
        d = fmaf(o[n].x, g.x, fmaf(o[n].y, g.y, fmaf(o[n].z, g.z, fmaf(o[n].w, g.w, d))));
      }
    } else if (row != nullptr) {
      for (int e = part; e < hd; e += N) d = fmaf(to_f32(row[e]), sg[r * P + e], d);
    }
#pragma unroll
    for (int m = N / 2; m > 0; m >>= 1) d += __shfl_xor_sync(0xffffffffu, d, m);
    if (part == 0) dot[r] = d;
  }
};

template <typename T, int HD, int RB>
__device__ __forceinline__ void grad_queries(const Args& a, bool quads, float* sm, uint32_t* bad, int* start, float* lse2, float* dot, int unit) {
  using W = Way<HD, RB>;
  float* sq = sm;
  float* sg = sq + W::rows;
  float* sk = sg + W::rows;
  float* sv = sk + W::block;
  float* sp = sv + W::block;
  const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15, hd = a.head_dim;
  const int tiles = (int)((a.tokens + W::B - 1) / W::B);
  const int head = unit % a.heads, rest = unit / a.heads, rep = rest % a.m;
  const int64_t r0 = (int64_t)(tiles - 1 - rest / a.m) * W::B;
  const int kvh = head / (a.heads / a.kv_heads);
  const int64_t stat = ((int64_t)rep * a.heads + head) * a.tokens;
  RowDots<T, W, HD, W::B> dots_of_rows;
  dots_of_rows.fetch(head_ptr<const T>(a.out, rep, head, hd), a.out.row, r0, a.tokens, hd, quads);
  load_two<T, W, HD, W::B>(sq, head_ptr<const T>(a.q, rep, head, hd), a.q.row, sg, head_ptr<const T>(a.dout, rep, head, hd), a.dout.row, r0,
                           a.tokens, hd, quads);
  const Bounds bounds(a, rep);
  if (tid < W::B) {                        // (whole warps)
    int end;
    bad[tid] = 0u;
    bounds.rows((int)r0 + (tid & ~31), &start[tid], &end);
    lse2[tid] = r0 + tid < a.tokens ? a.lse[stat + r0 + tid] * kLog2e : 0.f;
  }
  __syncthreads();
  dots_of_rows.finish(dot, sg, hd, quads);
  const float scale2 = a.scale * kLog2e;
  float acc[W::R][W::C] = {};
  const int64_t end = min(r0 + W::B, a.tokens);
  for (int64_t j0 = bounds.first_key((int)r0); j0 < end; j0 += W::N) {
    load_two<T, W, HD, W::N>(sk, head_ptr<const T>(a.k, rep, kvh, hd), a.k.row, sv, head_ptr<const T>(a.v, rep, kvh, hd), a.v.row, j0, a.tokens,
                             hd, quads);
    __syncthreads();
    float s[W::R][W::K], g[W::R][W::K];
    dots<W, HD>(sq, sk, ty, tx, s);
    dots<W, HD>(sg, sv, ty, tx, g);
#pragma unroll
    for (int r = 0; r < W::R; ++r) {
      const int row = ty * W::R + r;
#pragma unroll
      for (int c = 0; c < W::K; ++c) {
        const int64_t j = j0 + tx + 16 * c;
        const bool seen = j >= start[row] && j <= r0 + row;
        sp[row * W::PS + tx + 16 * c] = seen ? exp2f(fmaf(s[r][c], scale2, -lse2[row])) * (g[r][c] - dot[row]) : 0.f;
      }
    }
    __syncwarp();                          // (a row of scores is one half warp's)
    accumulate<W, HD>(sp, sk, ty, tx, acc);
    __syncthreads();
  }
  float by[W::R];
#pragma unroll
  for (int r = 0; r < W::R; ++r) {
    by[r] = a.scale;
    if (start[ty * W::R + r] > r0 + ty * W::R + r) {
#pragma unroll
      for (int c = 0; c < W::C; ++c) acc[r][c] = 0.f;
    }
  }
  const bool good = write_rows<T, W, HD>(head_ptr<T>(a.dq, rep, head, hd), a.dq.row, r0, a.tokens, hd, ty, tx, acc, by, bad);
  if (__syncthreads_and(good)) return;
  const uint32_t ill = bad_rows<W>(bad);
  if (ill != 0u) dq_rows<T, HD / 32>(a, rep, head, (int)r0 + first_bad<W>(), ill);
}

// Tiles of keys: scores with the keys as rows and the queries as columns.  `rank` of the `split` CTAs that share the queries.
template <typename T, int HD, int RB>
__device__ __forceinline__ void grad_keys(const Args& a, bool quads, float* sm, uint32_t* bad, int* start, float* lse2, float* dot, int unit,
                                          int rank, int split) {
  using W = Way<HD, RB>;
  float* sk = sm;
  float* sv = sk + W::rows;
  float* sq = sv + W::rows;
  float* sg = sq + W::block;
  float* sp = sg + W::block;
  const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15, hd = a.head_dim;
  const int kvh = unit % a.kv_heads, rest = unit / a.kv_heads, rep = rest % a.m;
  const int64_t k0 = (int64_t)(rest / a.m) * W::B;
  const int group = a.heads / a.kv_heads;
  load_two<T, W, HD, W::B>(sk, head_ptr<const T>(a.k, rep, kvh, hd), a.k.row, sv, head_ptr<const T>(a.v, rep, kvh, hd), a.v.row, k0, a.tokens,
                           hd, quads);
  if (tid < W::B) bad[tid] = 0u;
  const float scale2 = a.scale * kLog2e;
  float dk[W::R][W::C] = {}, dv[W::R][W::C] = {};
  const Bounds bounds(a, rep);
  const int64_t end = bounds.last_query((int)min(k0 + W::B, a.tokens) - 1);
  // steps are tiles of queries, head by head; this CTA has its part of them
  const int per = end > k0 ? (int)((end - k0 + W::N - 1) / W::N) : 0;
  const int64_t all = (int64_t)per * group;
  for (int64_t step = all * rank / split; step < all * (rank + 1) / split; ++step) {
    const int head = kvh * group + (int)(step / per);
    const int64_t i0 = k0 + step % per * W::N, stat = ((int64_t)rep * a.heads + head) * a.tokens;
    __syncthreads();
    const float of_row = tid < W::N && i0 + tid < a.tokens ? a.lse[stat + i0 + tid] : 0.f;
    RowDots<T, W, HD, W::N> dots_of_rows;
    dots_of_rows.fetch(head_ptr<const T>(a.out, rep, head, hd), a.out.row, i0, a.tokens, hd, quads);
    load_two<T, W, HD, W::N>(sq, head_ptr<const T>(a.q, rep, head, hd), a.q.row, sg, head_ptr<const T>(a.dout, rep, head, hd), a.dout.row, i0,
                             a.tokens, hd, quads);
    if (tid < W::N) {
      int stop;
      lse2[tid] = of_row * kLog2e;
      bounds.rows((int)i0 + (tid & ~31), &start[tid], &stop);
    }
    __syncthreads();
    dots_of_rows.finish(dot, sg, hd, quads);
    float s[W::R][W::K], g[W::R][W::K];
    dots<W, HD>(sk, sq, ty, tx, s);
    dots<W, HD>(sv, sg, ty, tx, g);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < W::R; ++r) {
      const int64_t j = k0 + ty * W::R + r;
#pragma unroll
      for (int c = 0; c < W::K; ++c) {
        const int col = tx + 16 * c;
        const bool seen = j >= start[col] && j <= i0 + col;
        const float p = seen ? exp2f(fmaf(s[r][c], scale2, -lse2[col])) : 0.f;
        sp[(ty * W::R + r) * W::PS + col] = p;
        s[r][c] = seen ? p * (g[r][c] - dot[col]) : 0.f;
      }
    }
    __syncwarp();                        // (a row of scores is one half warp's)
    accumulate<W, HD>(sp, sg, ty, tx, dv);
    __syncwarp();
#pragma unroll
    for (int r = 0; r < W::R; ++r)
#pragma unroll
      for (int c = 0; c < W::K; ++c) sp[(ty * W::R + r) * W::PS + tx + 16 * c] = s[r][c];
    __syncwarp();
    accumulate<W, HD>(sp, sq, ty, tx, dk);
  }
  if (split > 1) {
    // a thread's numbers beside those of the other threads, so that neighbours read neighbouring words
    __syncthreads();
    if (rank > 0) {
#pragma unroll
      for (int r = 0; r < W::R; ++r)
#pragma unroll
        for (int c = 0; c < W::C; ++c) {
          sm[(r * W::C + c) * W::NT + tid] = dk[r][c];
          sm[((W::R + r) * W::C + c) * W::NT + tid] = dv[r][c];
        }
    }
    ptx::cluster_sync_all();
    if (rank == 0) {
      for (int p = 1; p < split; ++p) {
        const uint32_t at = ptx::map_to_rank(ptx::smem_u32(sm + tid), p);
#pragma unroll
        for (int r = 0; r < W::R; ++r)
#pragma unroll
          for (int c = 0; c < W::C; ++c) {
            dk[r][c] += ptx::ld_cluster_f32(at + (r * W::C + c) * W::NT * 4);
            dv[r][c] += ptx::ld_cluster_f32(at + ((W::R + r) * W::C + c) * W::NT * 4);
          }
      }
    }
    ptx::cluster_sync_all();               // (the others' shared memory has been read)
    if (rank > 0) return;
  }
  float one[W::R], scale[W::R];
#pragma unroll
  for (int r = 0; r < W::R; ++r) { one[r] = 1.f; scale[r] = a.scale; }
  bool good = write_rows<T, W, HD>(head_ptr<T>(a.dk, rep, kvh, hd), a.dk.row, k0, a.tokens, hd, ty, tx, dk, scale, bad);
  good = write_rows<T, W, HD>(head_ptr<T>(a.dv, rep, kvh, hd), a.dv.row, k0, a.tokens, hd, ty, tx, dv, one, bad) && good;
  if (__syncthreads_and(good)) return;
  const uint32_t ill = bad_rows<W>(bad);
  if (ill != 0u) dkv_rows<T, HD / 32>(a, rep, kvh, (int)k0 + first_bad<W>(), ill, nullptr);
}

// The first `key_units` times `split` CTAs have tiles of keys (those with the most queries first), the others tiles of queries (those
// with the most keys first).
template <typename T, int HD, int RB>
__global__ void __launch_bounds__(Way<HD, RB>::NT, least_ctas<HD, RB>(true))
attention_grad_kernel(const __grid_constant__ Args a, const bool quads, const int key_units, const int query_units, const int split) {
  using W = Way<HD, RB>;
  extern __shared__ __align__(16) float sm[];
  __shared__ uint32_t bad[W::B];
  constexpr int M = W::B > W::N ? W::B : W::N;
  __shared__ float lse2[M], dot[M];
  __shared__ int start[M];
  grid_dep_wait();
  grid_dep_launch();
  const int unit = (int)blockIdx.x / split;
  if (unit < key_units) {
    grad_keys<T, HD, RB>(a, quads, sm, bad, start, lse2, dot, unit, (int)blockIdx.x % split, split);
  } else {
    const int query = (int)blockIdx.x - key_units * split;
    if (query < query_units) grad_queries<T, HD, RB>(a, quads, sm, bad, start, lse2, dot, query);
  }
}

// fours of elements: their rows, heads and replicas start on a boundary of 16 (bf16: 8) bytes
template <typename T>
bool whole_quads(const Args& a) {
  if (a.head_dim % 4 != 0) return false;
  for (const Tensor* t : {&a.q, &a.k, &a.v, &a.out, &a.dout})
    if (t->p != nullptr && (reinterpret_cast<uintptr_t>(t->p) % (4 * sizeof(T)) != 0 || t->row % 4 != 0 || t->replica % 4 != 0)) return false;
  return true;
}
// How many CTAs share the queries of a tile of keys: as many, up to eight, as still find an SM, two to each, or one where the shared
// memory leaves room for one (1000 rows of 4 heads of 200 on 1: 604 us with 256 such CTAs, 468 with 128).
int query_split(int64_t key_units, int per_sm) {
  int split = 1;
  while (split < 8 && key_units * split * 2 <= per_sm * 148) split *= 2;
  return split;
}

template <typename T, int HD, int RB>
cudaError_t launch(const Args& a, bool grad, cudaStream_t st) {
  using W = Way<HD, RB>;
  constexpr int fwd = (W::rows + 2 * W::block + W::scores) * 4, bwd = (2 * W::rows + 2 * W::block + W::scores) * 4;
  static_assert(bwd <= 220 * 1024, "shared memory budget");
  static_assert(2 * W::R * W::C * W::NT <= 2 * W::rows + 2 * W::block, "the parts of a cluster");
  static uint64_t done[2] = {0, 0};      // one bit per device
  const int64_t tiles = (a.tokens + W::B - 1) / W::B;
  const bool quads = whole_quads<T>(a);
  if (!grad) {
    const cudaError_t e = allow_dynamic_smem(attention_kernel<T, HD, RB>, fwd, &done[0]);
    if (e != cudaSuccess) return e;
    return launch_dep(attention_kernel<T, HD, RB>, dim3((unsigned)(tiles * a.heads * a.m)), dim3(W::NT), fwd, st, 1, a, quads);
  }
  const cudaError_t e = allow_dynamic_smem(attention_grad_kernel<T, HD, RB>, bwd, &done[1]);
  if (e != cudaSuccess) return e;
  const int64_t key_units = tiles * a.kv_heads * a.m, query_units = tiles * a.heads * a.m;
  const int split = query_split(key_units, HD > 128 ? 1 : 2);
  const int64_t ctas = key_units * split + (query_units + split - 1) / split * split;
  return launch_dep(attention_grad_kernel<T, HD, RB>, dim3((unsigned)ctas), dim3(W::NT), bwd, st, (unsigned)split, a, quads,
                    (int)key_units, (int)query_units, split);
}
// Tiles of 64 rows, or of 32 where those would leave SMs without one: a tile's blocks of keys follow one another, and half the rows
// take about half the time.
template <typename T, int HD>
cudaError_t pick_rows(const Args& a, bool grad, cudaStream_t st) {
  const bool few = (a.tokens + 63) / 64 * a.heads * a.m <= 148;
  return few ? launch<T, HD, 32>(a, grad, st) : launch<T, HD, 64>(a, grad, st);
}
template <typename T>
cudaError_t pick(const Args& a, bool grad, cudaStream_t st) {
  if (a.head_dim <= 32) return pick_rows<T, 32>(a, grad, st);
  if (a.head_dim <= 64) return pick_rows<T, 64>(a, grad, st);
  if (a.head_dim <= 128) return pick_rows<T, 128>(a, grad, st);
  return launch<T, 256, 32>(a, grad, st);
}
cudaError_t run(const Args& a, int dtype, bool grad, cudaStream_t st) {
  return dtype == LS_DTYPE_BF16 ? pick<__nv_bfloat16>(a, grad, st) : pick<float>(a, grad, st);
}

// ---- host side ---------------------------------------------------------------------------------------------------

int check_sizes(int m, int64_t tokens, int heads, int kv_heads, int head_dim, int dtype) {
  if (m < 1 || tokens < 0 || heads < 1 || kv_heads < 1 || heads % kv_heads != 0 || head_dim < 1) return LS_ERR_INVALID_ARG;
  if (dtype != LS_DTYPE_FP32 && dtype != LS_DTYPE_BF16) return LS_ERR_INVALID_ARG;
  if (m > 65535 || tokens > (1ll << 30) || heads > 65536 || head_dim > 256) return LS_ERR_TOO_LARGE;
  // (tiles of 32 rows, all heads, all replicas, of queries and keys: blocks of one launch)
  if ((tokens + 31) / 32 * heads > 1073741823ll / m) return LS_ERR_TOO_LARGE;
  return LS_OK;
}
// distances that no element uses, as the kernels' tensor maps take them
void settle(const Args& a, Tensor* t, int heads) {
  if (a.tokens <= 1) t->row = (int64_t)heads * a.head_dim;
  if (a.m == 1) t->replica = a.tokens * t->row;
}
// a tensor [m][tokens][heads][head_dim] whose rows are dense
bool bad_tensor(const Args& a, const Tensor& t, int heads, int dtype) {
  const int64_t width = (int64_t)heads * a.head_dim;
  if (reinterpret_cast<uintptr_t>(t.p) % (dtype == LS_DTYPE_BF16 ? 2 : 4) != 0) return true;
  if (a.tokens == 0) return false;
  if (t.p == nullptr || (a.tokens > 1 && t.row < width)) return true;
  if (t.row > (1ll << 40) / a.tokens) return true;
  return a.m > 1 && t.replica < (a.tokens - 1) * (a.tokens > 1 ? t.row : 0) + width;
}
bool misaligned4(const void* p) { return reinterpret_cast<uintptr_t>(p) % 4 != 0; }

}  // namespace
}  // namespace attn
}  // namespace ls

extern "C" int ls_attention(const void* q_dev, const void* k_dev, const void* v_dev, const int32_t* seq_start_dev, int m,
                            int64_t tokens, int n_seqs, int heads, int kv_heads, int head_dim, int64_t q_row, int64_t k_row,
                            int64_t v_row, int64_t q_stride, int64_t k_stride, int64_t v_stride, int dtype, float scale,
                            void* out_dev, int64_t out_row, int64_t out_stride, float* lse_dev, void* cuda_stream) {
  using namespace ls;
  using namespace ls::attn;
  int rc = check_sizes(m, tokens, heads, kv_heads, head_dim, dtype);
  if (rc != LS_OK) return rc;
  Args a{};
  a.m = m; a.tokens = tokens; a.heads = heads; a.kv_heads = kv_heads; a.head_dim = head_dim; a.n_seqs = n_seqs; a.scale = scale;
  a.q = Tensor{const_cast<void*>(q_dev), q_row, q_stride};
  a.k = Tensor{const_cast<void*>(k_dev), k_row, k_stride};
  a.v = Tensor{const_cast<void*>(v_dev), v_row, v_stride};
  a.out = Tensor{out_dev, out_row, out_stride};
  a.lse = lse_dev;
  a.seq_start = seq_start_dev;
  if (n_seqs < 0 || n_seqs > (1 << 30) || (seq_start_dev == nullptr && n_seqs != 1) || !isfinite(scale)) return LS_ERR_INVALID_ARG;
  if (bad_tensor(a, a.q, heads, dtype) || bad_tensor(a, a.k, kv_heads, dtype) || bad_tensor(a, a.v, kv_heads, dtype) ||
      bad_tensor(a, a.out, heads, dtype) || misaligned4(lse_dev) || misaligned4(seq_start_dev) ||
      (tokens > 0 && lse_dev == nullptr))
    return LS_ERR_INVALID_ARG;
  if (tokens == 0) return LS_OK;
  settle(a, &a.q, heads);
  settle(a, &a.out, heads);
  settle(a, &a.k, kv_heads);
  settle(a, &a.v, kv_heads);
  a.err = gop::device_error_word();
  if (a.err == nullptr) return LS_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  return (tc_takes(a, dtype) ? tc_forward(a, st) : run(a, dtype, false, st)) == cudaSuccess ? LS_OK : LS_ERR_CUDA;
}

extern "C" int ls_attention_grad_ws_bytes(int m, int64_t tokens, int heads, int kv_heads, int head_dim, size_t* bytes) {
  using namespace ls::attn;
  const int rc = check_sizes(m, tokens, heads, kv_heads, head_dim, LS_DTYPE_FP32);
  if (rc != LS_OK) return rc;
  if (bytes == nullptr) return LS_ERR_INVALID_ARG;
  *bytes = (size_t)m * (size_t)heads * (size_t)tokens * sizeof(float);
  return LS_OK;
}

extern "C" int ls_attention_grad(const void* dout_dev, const void* q_dev, const void* k_dev, const void* v_dev, const void* out_dev,
                                 const float* lse_dev, const int32_t* seq_start_dev, int m, int64_t tokens, int n_seqs, int heads,
                                 int kv_heads, int head_dim, int64_t dout_row, int64_t q_row, int64_t k_row, int64_t v_row,
                                 int64_t out_row, int64_t dout_stride, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                                 int64_t out_stride, int dtype, float scale, void* dq_dev, void* dk_dev, void* dv_dev, int64_t dq_row,
                                 int64_t dk_row, int64_t dv_row, int64_t dq_stride, int64_t dk_stride, int64_t dv_stride,
                                 void* ws_dev, size_t ws_bytes, void* cuda_stream) {
  using namespace ls;
  using namespace ls::attn;
  int rc = check_sizes(m, tokens, heads, kv_heads, head_dim, dtype);
  if (rc != LS_OK) return rc;
  Args a{};
  a.m = m; a.tokens = tokens; a.heads = heads; a.kv_heads = kv_heads; a.head_dim = head_dim; a.n_seqs = n_seqs; a.scale = scale;
  a.dout = Tensor{const_cast<void*>(dout_dev), dout_row, dout_stride};
  a.q = Tensor{const_cast<void*>(q_dev), q_row, q_stride};
  a.k = Tensor{const_cast<void*>(k_dev), k_row, k_stride};
  a.v = Tensor{const_cast<void*>(v_dev), v_row, v_stride};
  a.out = Tensor{const_cast<void*>(out_dev), out_row, out_stride};
  a.dq = Tensor{dq_dev, dq_row, dq_stride};
  a.dk = Tensor{dk_dev, dk_row, dk_stride};
  a.dv = Tensor{dv_dev, dv_row, dv_stride};
  a.lse = const_cast<float*>(lse_dev);
  a.seq_start = seq_start_dev;
  if (n_seqs < 0 || n_seqs > (1 << 30) || (seq_start_dev == nullptr && n_seqs != 1) || !isfinite(scale)) return LS_ERR_INVALID_ARG;
  for (const Tensor* t : {&a.dout, &a.q, &a.out, &a.dq})
    if (bad_tensor(a, *t, heads, dtype)) return LS_ERR_INVALID_ARG;
  for (const Tensor* t : {&a.k, &a.v, &a.dk, &a.dv})
    if (bad_tensor(a, *t, kv_heads, dtype)) return LS_ERR_INVALID_ARG;
  if (misaligned4(lse_dev) || misaligned4(seq_start_dev) || (tokens > 0 && lse_dev == nullptr)) return LS_ERR_INVALID_ARG;
  if (ws_dev == nullptr && tokens > 0) return LS_ERR_INVALID_ARG;
  size_t need = 0;
  rc = ls_attention_grad_ws_bytes(m, tokens, heads, kv_heads, head_dim, &need);
  if (rc != LS_OK) return rc;
  if (ws_bytes < need || reinterpret_cast<uintptr_t>(ws_dev) % 256 != 0) return LS_ERR_STATE_SIZE;
  if (tokens == 0) return LS_OK;
  for (Tensor* t : {&a.dout, &a.q, &a.out, &a.dq}) settle(a, t, heads);
  for (Tensor* t : {&a.k, &a.v, &a.dk, &a.dv}) settle(a, t, kv_heads);
  a.dot = static_cast<float*>(ws_dev);
  a.err = gop::device_error_word();
  if (a.err == nullptr) return LS_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  return (tc_takes(a, dtype) ? tc_backward(a, st) : run(a, dtype, true, st)) == cudaSuccess ? LS_OK : LS_ERR_CUDA;
}
