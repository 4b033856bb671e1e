// The global norm of every replica's gradients over many tensors, and clipping to it (ls_clip_grads).
//
//   norm_r = sqrt( sum over the tensors of replica r of g^2 ),   out = g if norm_r <= max_norm, else g * (max_norm / norm_r)
//
// Two launches whatever the number of tensors (up to kClipMost; more take more): the first reads everything once and leaves one
// sum a CTA, the second adds the CTAs' sums in index order, redundantly in every CTA (a few hundred numbers), and scales.
// Where nothing is clipped in place it ends there.  Bound by HBM.  A replica's tensors are one sequence of chunks of 8192
// elements, of which every CTA takes a run; the second launch takes its run backwards, so that what the first one read last is
// still in the L2 (126 MB): two replicas of 332 million fp32 elements into bf16 in 383 + 631 us, 7.0 and 6.3 TB/s of what each launch
// reads and writes; 38 tensors of four small replicas, whose second launch has nothing to scale, in 23 + 5 us.
//
// Squares are added in fp32 over the 32 elements that a thread has of a chunk, and in double beyond.  Where such a sum
// overflows or comes near the smallest fp32 numbers, the 32 squares are added once more in double.
#include "ls_internal.h"

#include <math.h>
#include <string.h>

#include <algorithm>
#include <new>
#include <vector>

namespace ls {
namespace {

constexpr int kClipChunk = 8192, kClipNT = 256;
constexpr int kClipFew = 64, kClipMost = 500;                // tensors of a launch: 3 KB or 24 KB of kernel arguments
constexpr int kClipPerSm = 4;

enum { CLIP_IN_BF16 = 1, CLIP_OUT_BF16 = 2, CLIP_VEC = 4, CLIP_SAME = 8 };
struct ClipTensor {
  const void* in;
  void* out;
  int64_t in_stride, out_stride, n;
  int32_t first;                         // of its chunks
  int32_t flags;
};
template <int MOST>
struct ClipArgs {
  int count, chunks, parts;              // tensors and chunks of this launch; CTAs' sums of a replica over all launches
  int part0;                             // where this launch's are
  double* part;                          // [m][parts]
  double max_norm;
  float* norm;
  ClipTensor t[MOST];
};

__device__ __forceinline__ void clip_load8(const void* p, int64_t at, bool bf16, float (&x)[8]) {
  if (bf16) {
    const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p) + at);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
  } else {
    const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
    const float4 a = q[0], b = q[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
}
__device__ __forceinline__ void clip_store8(void* p, int64_t at, bool bf16, const float (&x)[8]) {
  if (bf16) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p) + at) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
    float4* q = reinterpret_cast<float4*>(static_cast<float*>(p) + at);
    q[0] = make_float4(x[0], x[1], x[2], x[3]);
    q[1] = make_float4(x[4], x[5], x[6], x[7]);
  }
}
__device__ __forceinline__ float clip_load(const void* p, int64_t at, bool bf16) {
  return bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[at]) : static_cast<const float*>(p)[at];
}
__device__ __forceinline__ void clip_store(void* p, int64_t at, bool bf16, float x) {
  if (bf16) static_cast<__nv_bfloat16*>(p)[at] = __float2bfloat16_rn(x);
  else static_cast<float*>(p)[at] = x;
}

// A thread's 32 elements of a chunk: four pieces of eight (vectors), or every 256th element.
__device__ __forceinline__ void clip_chunk(const ClipTensor& t, int64_t rep, int64_t at, float (&x)[4][8]) {
  const bool bf16 = (t.flags & CLIP_IN_BF16) != 0;
  const char* base = static_cast<const char*>(t.in) + rep * t.in_stride * (bf16 ? 2 : 4);
  if ((t.flags & CLIP_VEC) != 0 && at + kClipChunk <= t.n) {
#pragma unroll
    for (int u = 0; u < 4; ++u) clip_load8(base, at + (u * kClipNT + threadIdx.x) * 8, bf16, x[u]);
  } else {
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int64_t i = at + (u * 8 + e) * kClipNT + threadIdx.x;
        x[u][e] = i < t.n ? clip_load(base, i, bf16) : 0.f;
      }
  }
}

__device__ __forceinline__ double clip_block_sum(double s, double* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
  __syncthreads();
  double t = 0.0;
#pragma unroll
  for (int w = 0; w < kClipNT / 32; ++w) t += red[w];
  return t;
}

template <int MOST>
__device__ __forceinline__ int clip_find(const ClipArgs<MOST>& a, int chunk) {
  int lo = 0, hi = a.count - 1;          // the last tensor whose first chunk is <= chunk
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.t[mid].first <= chunk) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

template <int MOST>
__global__ void __launch_bounds__(kClipNT)
clip_norm_kernel(const __grid_constant__ ClipArgs<MOST> a) {
  __shared__ double red[kClipNT / 32];
  grid_dep_wait();
  grid_dep_launch();
  const int64_t rep = blockIdx.y;
  const int c0 = (int)((int64_t)a.chunks * blockIdx.x / gridDim.x), c1 = (int)((int64_t)a.chunks * (blockIdx.x + 1) / gridDim.x);
  double total = 0.0;
  int k = c0 < c1 ? clip_find(a, c0) : 0;
  for (int c = c0; c < c1; ++c) {
    while (k + 1 < a.count && a.t[k + 1].first <= c) ++k;
    float x[4][8];
    clip_chunk(a.t[k], rep, (int64_t)(c - a.t[k].first) * kClipChunk, x);
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) s[u] = fmaf(x[u][e], x[u][e], s[u]);
    const float sum = (s[0] + s[1]) + (s[2] + s[3]);
    if (sum > 1e-30f && sum < 1e38f) {
      total += (double)sum;
    } else {
      // out of fp32's range, or zeros, of which there may be many
      uint32_t any = 0;
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) any |= __float_as_uint(x[u][e]) << 1;
      if (any != 0)
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int e = 0; e < 8; ++e) total = fma((double)x[u][e], (double)x[u][e], total);
    }
  }
  total = clip_block_sum(total, red);
  if (threadIdx.x == 0) a.part[rep * a.parts + a.part0 + blockIdx.x] = total;
}

template <int MOST>
__global__ void __launch_bounds__(kClipNT)
clip_scale_kernel(const __grid_constant__ ClipArgs<MOST> a) {
  __shared__ double red[kClipNT / 32];
  grid_dep_wait();
  grid_dep_launch();
  const int64_t rep = blockIdx.y;
  double total = 0.0;
  for (int i = threadIdx.x; i < a.parts; i += kClipNT) total += __ldcg(a.part + rep * a.parts + i);
  const double norm = sqrt(clip_block_sum(total, red));
  if (blockIdx.x == 0 && threadIdx.x == 0) a.norm[rep] = (float)norm;
  const bool clips = !(norm <= a.max_norm) && a.max_norm < INFINITY;       // (a norm of NaN makes everything NaN)
  // The factor; one far below 1 (10^-76 where norm and limit are at fp32's ends) in two, a power of two of half its order taken
  // first, so that neither the factors nor the product between them leave fp32's range before the result does.
  const double factor = clips ? a.max_norm / norm : 1.0;
  const int half = factor > 0.0 && factor < 1e-30 ? ilogb(factor) / 2 : 0;
  const float before = (float)ldexp(1.0, half), by = (float)ldexp(factor, -half);
  const int c0 = (int)((int64_t)a.chunks * blockIdx.x / gridDim.x), c1 = (int)((int64_t)a.chunks * (blockIdx.x + 1) / gridDim.x);
  int k = c0 < c1 ? clip_find(a, c1 - 1) : 0;
  for (int c = c1 - 1; c >= c0; --c) {
    while (a.t[k].first > c) --k;
    const ClipTensor& t = a.t[k];
    if (!clips && (t.flags & CLIP_SAME) != 0) continue;
    const int64_t at = (int64_t)(c - t.first) * kClipChunk;
    float x[4][8];
    clip_chunk(t, rep, at, x);
    const bool bf16 = (t.flags & CLIP_OUT_BF16) != 0;
    char* base = static_cast<char*>(t.out) + rep * t.out_stride * (bf16 ? 2 : 4);
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[u][e] = x[u][e] * before * by;
    if ((t.flags & CLIP_VEC) != 0 && at + kClipChunk <= t.n) {
#pragma unroll
      for (int u = 0; u < 4; ++u) clip_store8(base, at + (u * kClipNT + threadIdx.x) * 8, bf16, x[u]);
    } else {
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int64_t i = at + (u * 8 + e) * kClipNT + threadIdx.x;
          if (i < t.n) clip_store(base, i, bf16, x[u][e]);
        }
    }
  }
}

// ---- host side ---------------------------------------------------------------------------------------------------

struct ClipList {
  const void* const* in;
  void* const* out;
  const int64_t *n, *in_stride, *out_stride;
  const int32_t *in_dtype, *out_dtype;
  int count, m;
};
int64_t clip_chunks(int64_t n) { return (n + kClipChunk - 1) / kClipChunk; }
// CTAs of a replica in a launch of so many chunks
int clip_ctas(int64_t chunks, int m) {
  const int64_t most = (148 * kClipPerSm + m - 1) / m;
  return (int)(chunks < 1 ? 1 : chunks < most ? chunks : most);
}

// The tensors from `from` on that one launch takes; empty ones are left out.
template <int MOST>
int clip_fill(const ClipList& l, int from, ClipArgs<MOST>* a) {
  a->count = a->chunks = 0;
  int i = from;
  for (; i < l.count && a->count < MOST; ++i) {
    if (l.n[i] == 0) continue;
    ClipTensor& t = a->t[a->count++];
    t.in = l.in[i];
    t.out = l.out != nullptr ? l.out[i] : const_cast<void*>(l.in[i]);
    t.n = l.n[i];
    t.in_stride = l.m > 1 ? l.in_stride[i] : 0;
    t.out_stride = l.m > 1 ? (l.out != nullptr ? l.out_stride[i] : l.in_stride[i]) : 0;
    const bool ib = l.in_dtype[i] == LS_DTYPE_BF16, ob = l.out != nullptr ? l.out_dtype[i] == LS_DTYPE_BF16 : ib;
    const bool vec = reinterpret_cast<uintptr_t>(t.in) % 16 == 0 && reinterpret_cast<uintptr_t>(t.out) % 16 == 0 &&
                     t.in_stride % (ib ? 8 : 4) == 0 && t.out_stride % (ob ? 8 : 4) == 0;
    const bool same = t.out == t.in;
    t.flags = (ib ? CLIP_IN_BF16 : 0) | (ob ? CLIP_OUT_BF16 : 0) | (vec ? CLIP_VEC : 0) | (same ? CLIP_SAME : 0);
    t.first = a->chunks;
    a->chunks += (int)clip_chunks(t.n);
  }
  return i;
}

template <int MOST>
int clip_run(const ClipList& l, double max_norm, float* norm, double* part, int parts, cudaStream_t st) {
  ClipArgs<MOST> a;
  a.parts = parts;
  a.part = part;
  a.max_norm = max_norm;
  a.norm = norm;
  const bool only_norm = isinf(max_norm) && l.out == nullptr;
  for (int pass = 0; pass < 2; ++pass) {
    a.part0 = 0;
    int from = 0;
    do {                                  // (once at least: the norm of nothing is written, too)
      from = clip_fill(l, from, &a);
      int ctas = clip_ctas(a.chunks, l.m);
      cudaError_t e;
      if (pass == 0) {
        e = launch_dep(clip_norm_kernel<MOST>, dim3((unsigned)ctas, (unsigned)l.m), dim3(kClipNT), 0, st, 1, a);
      } else {
        if (only_norm) {
          from = l.count;
          a.chunks = 0;
          ctas = 1;
        }
        e = launch_dep(clip_scale_kernel<MOST>, dim3((unsigned)ctas, (unsigned)l.m), dim3(kClipNT), 0, st, 1, a);
      }
      if (e != cudaSuccess) return LS_ERR_CUDA;
      a.part0 += ctas;
    } while (from < l.count);
  }
  return LS_OK;
}

// Where a tensor's replicas lie: m pieces of `bytes`, `step` apart, from `at` on.  `out`: it is written.
struct ClipSpan {
  uint64_t at, step, bytes;
  bool out;
};
// Pieces in the order of their addresses, one after another: whether one that is written shares memory with another one.
struct ClipSweep {
  uint64_t read_end = 0, written_end = 0;
  bool meets(uint64_t at, const ClipSpan& s) {
    const bool hit = at < written_end || (s.out && at < read_end);
    uint64_t& end = s.out ? written_end : read_end;
    end = std::max(end, at + s.bytes);
    return hit;
  }
};
// Whether spans [from, to), in the order of their first pieces and within `extent` bytes, have a piece that is written and meets another.
bool clip_meet(const ClipSpan* from, const ClipSpan* to, uint64_t extent, int m) {
  const uint64_t step = from->step;
  bool same = true;
  for (const ClipSpan* s = from; s < to; ++s) same = same && s->step == step && s->at - from->at + s->bytes <= step;
  if (m == 1 || (same && extent <= step * (uint64_t)m)) {                    // views of replica vectors: replicas lie alike
    ClipSweep sweep;
    for (const ClipSpan* s = from; s < to; ++s)
      if (sweep.meets(s->at, *s)) return true;
    return false;
  }
  // others: all pieces, by a heap of every span's next one
  struct Next { uint64_t at; const ClipSpan* s; int rep; };
  std::vector<Next> heap;
  const auto later = [](const Next& a, const Next& b) { return a.at > b.at; };
  for (const ClipSpan* s = from; s < to; ++s) heap.push_back(Next{s->at, s, 0});
  std::make_heap(heap.begin(), heap.end(), later);
  ClipSweep sweep;
  while (!heap.empty()) {
    std::pop_heap(heap.begin(), heap.end(), later);
    Next& n = heap.back();
    if (sweep.meets(n.at, *n.s)) return true;
    if (++n.rep == m) {
      heap.pop_back();
    } else {
      n.at += n.s->step;
      std::push_heap(heap.begin(), heap.end(), later);
    }
  }
  return false;
}
// Whether an output shares memory with another output, or with a gradient that is not its own: CTAs would write what others still read.
// A gradient that is its own output, as it lies, is one span.  Spans whose extents do not overlap (tensors of their own) are
// told apart by one sort: 1 us for 38 tensors.  May throw std::bad_alloc.
bool clip_overlap(const ClipList& l) {
  std::vector<ClipSpan> spans;
  spans.reserve(2 * (size_t)l.count);
  const auto add = [&](const void* p, int64_t n, int64_t stride, int32_t dtype, bool out) {
    const uint64_t e = dtype == LS_DTYPE_BF16 ? 2 : 4;
    spans.push_back(ClipSpan{reinterpret_cast<uintptr_t>(p), l.m > 1 ? (uint64_t)std::min<int64_t>(stride, 1ll << 44) * e : 0, (uint64_t)n * e, out});
  };
  for (int i = 0; i < l.count; ++i) {
    if (l.n[i] == 0) continue;
    const bool own = l.out == nullptr || l.out[i] == l.in[i];
    add(l.in[i], l.n[i], l.m > 1 ? l.in_stride[i] : 0, l.in_dtype[i], own);
    if (!own) add(l.out[i], l.n[i], l.m > 1 ? l.out_stride[i] : 0, l.out_dtype[i], true);
  }
  std::sort(spans.begin(), spans.end(), [](const ClipSpan& a, const ClipSpan& b) { return a.at < b.at; });
  const auto end_of = [&](const ClipSpan& s) { return s.at + (uint64_t)(l.m - 1) * s.step + s.bytes; };
  for (size_t i = 0; i < spans.size();) {
    uint64_t end = end_of(spans[i]);
    size_t j = i + 1;
    for (; j < spans.size() && spans[j].at < end; ++j) end = std::max(end, end_of(spans[j]));
    if (j > i + 1 && clip_meet(&spans[i], &spans[i] + (j - i), end - spans[i].at, l.m)) return true;
    i = j;
  }
  return false;
}

// CTAs' sums of a replica over all launches, or a refusal
int clip_parts(const int64_t* n, int count, int m, int* parts) {
  if (m < 1 || count < 0 || (count > 0 && n == nullptr)) return LS_ERR_INVALID_ARG;
  for (int i = 0; i < count; ++i)
    if (n[i] < 0) return LS_ERR_INVALID_ARG;
  if (m > 65535 || count > 65536) return LS_ERR_TOO_LARGE;
  int live = 0;
  int64_t all = 0;
  for (int i = 0; i < count; ++i) {
    if (n[i] > (1ll << 40)) return LS_ERR_TOO_LARGE;
    live += n[i] > 0;
    all += clip_chunks(n[i]);
  }
  if (all > (1ll << 30)) return LS_ERR_TOO_LARGE;
  int launches = (live + kClipMost - 1) / kClipMost;
  if (launches < 1) launches = 1;
  *parts = launches * ((148 * kClipPerSm + m - 1) / m);
  return LS_OK;
}

}  // namespace
}  // namespace ls

extern "C" int ls_clip_grads_ws_bytes(const int64_t* sizes, int n_tensors, int m, size_t* bytes) {
  using namespace ls;
  int parts = 0;
  const int rc = clip_parts(sizes, n_tensors, m, &parts);
  if (rc != LS_OK) return rc;
  if (bytes == nullptr) return LS_ERR_INVALID_ARG;
  *bytes = (size_t)m * (size_t)parts * sizeof(double);
  return LS_OK;
}

extern "C" int ls_clip_grads(const void* const* grads_dev, const int64_t* sizes, const int64_t* strides, const int32_t* dtypes,
                             int n_tensors, int m, double max_norm, void* const* outs_dev, const int64_t* out_strides,
                             const int32_t* out_dtypes, float* norm_dev, void* ws_dev, size_t ws_bytes, void* cuda_stream) {
  using namespace ls;
  int parts = 0;
  const int rc = clip_parts(sizes, n_tensors, m, &parts);
  if (rc != LS_OK) return rc;
  if (!(max_norm > 0.0) || norm_dev == nullptr || reinterpret_cast<uintptr_t>(norm_dev) % 4 != 0 || ws_dev == nullptr) return LS_ERR_INVALID_ARG;
  if (n_tensors > 0 && (grads_dev == nullptr || dtypes == nullptr || (m > 1 && strides == nullptr))) return LS_ERR_INVALID_ARG;
  if (n_tensors > 0 && outs_dev != nullptr && (out_dtypes == nullptr || (m > 1 && out_strides == nullptr))) return LS_ERR_INVALID_ARG;
  auto bad = [&](const void* p, int64_t n, int32_t dtype, int64_t stride) {
    if (dtype != LS_DTYPE_FP32 && dtype != LS_DTYPE_BF16) return true;
    if (n == 0) return false;
    return p == nullptr || reinterpret_cast<uintptr_t>(p) % (dtype == LS_DTYPE_BF16 ? 2 : 4) != 0 || (m > 1 && stride < n);
  };
  for (int i = 0; i < n_tensors; ++i) {
    if (bad(grads_dev[i], sizes[i], dtypes[i], m > 1 ? strides[i] : 0)) return LS_ERR_INVALID_ARG;
    if (outs_dev == nullptr) continue;
    if (bad(outs_dev[i], sizes[i], out_dtypes[i], m > 1 ? out_strides[i] : 0)) return LS_ERR_INVALID_ARG;
    // (the tensor itself, as it lies, is the one output that may overlap its input)
    if (outs_dev[i] == grads_dev[i] && sizes[i] > 0 && (out_dtypes[i] != dtypes[i] || (m > 1 && out_strides[i] != strides[i])))
      return LS_ERR_INVALID_ARG;
  }
  if (ws_bytes < (size_t)m * (size_t)parts * sizeof(double) || reinterpret_cast<uintptr_t>(ws_dev) % 256 != 0) return LS_ERR_STATE_SIZE;
  while (n_tensors > 0 && sizes[n_tensors - 1] == 0) --n_tensors;          // (so that every launch has a tensor to read)
  const ClipList l{grads_dev, outs_dev, sizes, strides, out_strides, dtypes, out_dtypes, n_tensors, m};
  const bool only_norm = isinf(max_norm) && outs_dev == nullptr;             // (nothing is written, and tensors may share memory)
  try {
    if (!only_norm && clip_overlap(l)) return LS_ERR_INVALID_ARG;
  } catch (const std::bad_alloc&) {
    return LS_ERR_TOO_LARGE;
  }
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  double* part = static_cast<double*>(ws_dev);
  // the sums of all launches, whose CTAs may be fewer than there is room for
  int used = 0, live = 0;
  int64_t chunks = 0;
  const int most = [&] { int n = 0; for (int i = 0; i < n_tensors; ++i) n += sizes[i] > 0; return n; }() > kClipFew ? kClipMost : kClipFew;
  for (int i = 0; i < n_tensors; ++i) {
    if (sizes[i] == 0) continue;
    if (live == most) { used += clip_ctas(chunks, m); live = 0; chunks = 0; }
    ++live;
    chunks += clip_chunks(sizes[i]);
  }
  used += clip_ctas(chunks, m);
  return most == kClipMost ? clip_run<kClipMost>(l, max_norm, norm_dev, part, used, st) : clip_run<kClipFew>(l, max_norm, norm_dev, part, used, st);
}
