// Kernels that write pages of the 8-bit cache: append, compact, copy.
//
// Append and compact share one shape.  A CTA owns one page and one key/value head; its lower half of threads works on the
// keys, the upper half on the values.  It reads its rows once for the largest magnitude, settles the scale (a power of two,
// so that the division is exact and the only rounding is the one to e4m3), and reads them again, now from L1 or L2,
// for the codes.  Which sequence a CTA belongs to follows from cu_rows and the lengths on the device; the host sizes the grid
// for the most pages that so many rows can touch (rows / page + 2 per sequence), the CTAs beyond return at once.
#pragma once
#include "cache_common.cuh"

namespace ficoco {

constexpr int PAGE_THREADS = 256;
constexpr int PAGE_HALF = PAGE_THREADS / 2;

// Largest of `v` over the PAGE_HALF threads of each half of the CTA (all values >= 0).
__device__ __forceinline__ float half_max(float v, float (&warp_max)[PAGE_THREADS / 32]) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
  if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = v;
  __syncthreads();
  const float* m = warp_max + (threadIdx.x >= PAGE_HALF ? PAGE_HALF / 32 : 0);
  return fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
}

template <class T>
__global__ void __launch_bounds__(PAGE_THREADS) k_cache_append(const CacheView c, const T* __restrict__ k, const T* __restrict__ v,
                                                              const int* __restrict__ cu, long long k_stride, long long v_stride,
                                                              int rows, unsigned* __restrict__ status) {
  __shared__ float warp_max[PAGE_THREADS / 32];
  __shared__ int poisoned[128];
  grid_dep_wait();
  grid_dep_launch();
  const int u = blockIdx.x, head = blockIdx.y, tid = threadIdx.x;
  const int b = owner_of(c.batch, [&](int s) { return (long long)(max(cu[s], 0) >> c.log_page) + 2 * s; }, u);
  const int2 r = cache_rows(cu, b, rows, status);
  const int n = r.y - r.x, len = cache_length(c, b, status), start = len - n;
  if (n <= 0 || len <= 0) return;
  if (start < 0 && tid == 0) atomicOr(status, STATUS_CACHE);      // more rows than tokens: those in front are skipped
  const int from = max(start, 0);
  const int pi = (from >> c.log_page) + (u - ((max(cu[b], 0) >> c.log_page) + 2 * b));
  if (pi < from >> c.log_page || pi > (len - 1) >> c.log_page) return;
  const int page = cache_page(c, b, pi, -1, status);
  if (page < 0) return;
  const int s0 = max(from - (pi << c.log_page), 0), s1 = min(len - (pi << c.log_page), c.page);
  const int row0 = r.x + ((pi << c.log_page) + s0 - start);

  const bool is_v = tid >= PAGE_HALF;
  const int ht = tid & (PAGE_HALF - 1);
  const T* src = (is_v ? v : k) + (long long)row0 * (is_v ? v_stride : k_stride) + head * c.dim;
  const long long stride = is_v ? v_stride : k_stride;
  const size_t at = (size_t)page * c.kv + head;
  uint8_t* dst = (is_v ? c.v : c.k) + (at << c.log_page) * c.dim;
  float* scale = (is_v ? c.vs : c.ks) + at;
  const float old = s0 > 0 ? *scale : 0.f;
  const int vecs = c.dim >> 3, total = (s1 - s0) * vecs;       // vectors of eight elements

  if (tid < s1 - s0) poisoned[tid] = 0;
  __syncthreads();
  float amax = 0.f;
  bool bad = false;
  for (int i = ht; i < total; i += PAGE_HALF) {
    const int row = i / vecs;
    float f[8];
    load8(src + row * stride + (i - row * vecs) * 8, f);
    float m = 0.f, zero = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) { m = fmaxf(m, fabsf(f[j])); zero += f[j] * 0.f; }    // (NaN * 0 and infinity * 0 are NaN)
    if (zero != 0.f) { poisoned[row] = 1; bad = true; }
    amax = fmaxf(amax, m);
  }
  if (__syncthreads_or(bad)) {                                 // rare: once more without the rows that do not count
    amax = 0.f;
    for (int i = ht; i < total; i += PAGE_HALF) {
      const int row = i / vecs;
      if (poisoned[row]) continue;
      float f[8];
      load8(src + row * stride + (i - row * vecs) * 8, f);
#pragma unroll
      for (int j = 0; j < 8; ++j) amax = fmaxf(amax, fabsf(f[j]));
    }
  }
  amax = half_max(amax, warp_max);
  const float s = fmaxf(scale_of(amax), old), inv = 1.0f / s;
  if (s0 > 0 && s > old) {                                     // the older codes of the page move to the larger scale
    const float f = old * inv;
    for (int i = ht; i < s0 * vecs; i += PAGE_HALF) {
      uint2* p = reinterpret_cast<uint2*>(dst) + i;
      float x[8];
      from_e4m3x8(*p, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] *= f;
      *p = to_e4m3x8(x);
    }
  }
  uint2* out = reinterpret_cast<uint2*>(dst) + s0 * vecs;
  for (int i = ht; i < total; i += PAGE_HALF) {
    const int row = i / vecs;
    float f[8];
    load8(src + row * stride + (i - row * vecs) * 8, f);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] *= inv;
    uint2 codes = to_e4m3x8(f);
    if (poisoned[row]) codes = is_v ? make_uint2(0u, 0u) : make_uint2(E4M3_NAN4, E4M3_NAN4);
    out[i] = codes;
  }
  if (ht == 0) *scale = s;
}

__global__ void __launch_bounds__(PAGE_THREADS) k_cache_compact(const CacheView c, const int* __restrict__ to_table,
                                                               const int* __restrict__ kept, const int* __restrict__ cu,
                                                               int* __restrict__ lengths_out, long long to_stride,
                                                               int to_pages, int n_kept, int first,
                                                               unsigned* __restrict__ status) {
  __shared__ float warp_max[PAGE_THREADS / 32];
  __shared__ size_t row_at[128];                               // code offset of each row of the page in the pool
  __shared__ float row_scale[2][128];
  grid_dep_wait();
  grid_dep_launch();
  const int u = blockIdx.x, head = blockIdx.y, tid = threadIdx.x;
  auto unit0 = [&](int s) { return ((max(cu[s], 0) + (long long)s * first) >> c.log_page) + 2 * s; };
  const int b = owner_of(c.batch, unit0, u);
  const int2 r = cache_rows(cu, b, n_kept, status);
  const int len = cache_length(c, b, status), front = min(first, len), total_rows = front + (r.y - r.x);
  const int pi = (int)(u - unit0(b));
  if (pi == 0 && head == 0 && tid == 0 && lengths_out != nullptr) lengths_out[b] = total_rows;
  const int s1 = min(total_rows - (pi << c.log_page), c.page);
  if (pi < 0 || s1 <= 0) return;
  int page = -1;
  if (pi < to_pages) page = to_table[(long long)b * to_stride + pi];
  if ((unsigned)page >= (unsigned)c.n_pages) {
    if (tid == 0) atomicOr(status, STATUS_CACHE);
    return;
  }
  if (tid < s1) {
    const int i = (pi << c.log_page) + tid;
    int pos = i;
    if (i >= front) {
      const int e = kept[r.x + i - front];
      pos = front + e;
      if (e < 0 || pos >= len) { atomicOr(status, STATUS_CACHE); pos = 0; }
    }
    // a sequence without tokens has nothing to gather, not even token 0: zeros
    const int sp = len > 0 ? cache_page(c, b, pos >> c.log_page, 0, status) : 0;
    const size_t at = (size_t)sp * c.kv + head;
    row_at[tid] = ((at << c.log_page) + (pos & (c.page - 1))) * c.dim;
    row_scale[0][tid] = len > 0 ? c.ks[at] : 0.f;
    row_scale[1][tid] = len > 0 ? c.vs[at] : 0.f;
  }
  __syncthreads();
  const bool is_v = tid >= PAGE_HALF;
  const int ht = tid & (PAGE_HALF - 1);
  const uint8_t* src = is_v ? c.v : c.k;
  const float* rs = row_scale[is_v ? 1 : 0];
  const size_t at = (size_t)page * c.kv + head;
  const int vecs = c.dim >> 3, total = s1 * vecs;
  float amax = 0.f;
  for (int i = ht; i < total; i += PAGE_HALF) {
    const int row = i / vecs;
    float f[8];
    from_e4m3x8(*reinterpret_cast<const uint2*>(src + row_at[row] + (i - row * vecs) * 8), f);
    float m = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(f[j]));     // (a NaN key counts for nothing)
    amax = fmaxf(amax, m * rs[row]);
  }
  amax = half_max(amax, warp_max);
  const float s = scale_of(amax), inv = 1.0f / s;
  uint2* out = reinterpret_cast<uint2*>((is_v ? c.v : c.k) + (at << c.log_page) * c.dim);
  for (int i = ht; i < total; i += PAGE_HALF) {
    const int row = i / vecs;
    float f[8];
    from_e4m3x8(*reinterpret_cast<const uint2*>(src + row_at[row] + (i - row * vecs) * 8), f);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = (f[j] * rs[row]) * inv; // exact: powers of two (their quotient alone can overflow)
    out[i] = to_e4m3x8(f);
  }
  if (ht == 0) (is_v ? c.vs : c.ks)[at] = s;
}

// One CTA per page pair and part of the page; `words` 16-byte words of codes per page, keys and values alike.
constexpr int COPY_THREADS = 256;
__global__ void __launch_bounds__(COPY_THREADS) k_cache_copy(const CacheView c, const int* __restrict__ src,
                                                            const int* __restrict__ dst, int words,
                                                            unsigned* __restrict__ status) {
  grid_dep_wait();
  grid_dep_launch();
  const int from = src[blockIdx.x], to = dst[blockIdx.x];
  if (from < 0 || to < 0 || from == to) return;
  if (from >= c.n_pages || to >= c.n_pages) {
    if (threadIdx.x == 0) atomicOr(status, STATUS_CACHE);
    return;
  }
  const int per = (words + gridDim.y - 1) / gridDim.y, lo = blockIdx.y * per, hi = min(words, lo + per);
  for (int w = 0; w < 2; ++w) {
    const uint4* s = reinterpret_cast<const uint4*>(w ? c.v : c.k) + (size_t)from * words;
    uint4* d = reinterpret_cast<uint4*>(w ? c.v : c.k) + (size_t)to * words;
    int i = lo + threadIdx.x;
    for (; i + 3 * COPY_THREADS < hi; i += 4 * COPY_THREADS) {           // four loads in flight
      const uint4 a0 = s[i], a1 = s[i + COPY_THREADS], a2 = s[i + 2 * COPY_THREADS], a3 = s[i + 3 * COPY_THREADS];
      d[i] = a0; d[i + COPY_THREADS] = a1; d[i + 2 * COPY_THREADS] = a2; d[i + 3 * COPY_THREADS] = a3;
    }
    for (; i < hi; i += COPY_THREADS) d[i] = s[i];
    if (blockIdx.y == 0) {
      float* sc = w ? c.vs : c.ks;
      for (int h = threadIdx.x; h < c.kv; h += COPY_THREADS) sc[(size_t)to * c.kv + h] = sc[(size_t)from * c.kv + h];
    }
  }
}

}  // namespace ficoco
