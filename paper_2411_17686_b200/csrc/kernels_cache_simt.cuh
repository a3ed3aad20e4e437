// Attention over the 8-bit cache and its weights on the CUDA cores: any head size, one CTA per query row and head.
//
// A thread takes a token: its key's codes are read 16 at a time and multiplied with the query row, which lies in shared memory
// as fp32.  For the output a thread takes one or two dimensions and walks the tokens of the chunk.  What bounds it is arithmetic (a
// conversion and a multiplication per code and query row): the tensor-core kernels take head sizes of 64 and 128.  Measured where both can
// run: 64 ragged sequences of 64 to 8192 tokens, 32 heads on 8 of 128, 741 us (65 there); weights of 16 sequences 677 us (36).  Heads of 96: 683
// and 268 us, of 256: 925 us.
#pragma once
#include "cache_common.cuh"

namespace ficoco {

constexpr int CS_THREADS = 128;

__device__ __forceinline__ float dot16(const uint4& u, const float* q, float acc) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 a = from_e4m3x2(w[i] & 0xFFFFu), b = from_e4m3x2(w[i] >> 16);
    const float4 x = *reinterpret_cast<const float4*>(q + 4 * i);
    acc = fmaf(a.x, x.x, acc); acc = fmaf(a.y, x.y, acc); acc = fmaf(b.x, x.z, acc); acc = fmaf(b.y, x.w, acc);
  }
  return acc;
}

// Score of the query row in q (scaled to powers of two) with token j, in units of log2.
__device__ __forceinline__ float simt_score(const CacheView& c, int b, int kvh, int j, const float* q, unsigned* status) {
  const size_t at = (size_t)cache_page(c, b, j >> c.log_page, 0, status) * c.kv + kvh;
  const uint4* k = reinterpret_cast<const uint4*>(c.k + ((at << c.log_page) + (j & (c.page - 1))) * c.dim);
  float acc = 0.f;
  for (int i = 0; i < c.dim >> 4; ++i) acc = dot16(k[i], q + 16 * i, acc);
  return acc * c.ks[at];
}

template <class T>
__global__ void __launch_bounds__(CS_THREADS) k_cache_attention_simt(const CacheView c, const T* __restrict__ q,
                                                                    const int* __restrict__ cu, T* __restrict__ out,
                                                                    float* __restrict__ lse, long long q_stride, float scale_log2,
                                                                    int rows, int heads, const MaskRule mask,
                                                                    unsigned* __restrict__ status) {
  __shared__ __align__(16) float qs[256];
  __shared__ float ps[CS_THREADS], red[CS_THREADS / 32];
  __shared__ const uint8_t* vs_at[CS_THREADS];
  grid_dep_wait();
  grid_dep_launch();
  const int row = blockIdx.x, h = blockIdx.y, tid = threadIdx.x;
  const int b = owner_of(c.batch, [&](int s) { return (long long)cu[s]; }, row);
  const int2 r = cache_rows(cu, b, rows, status);
  if (row < r.x || row >= r.y) return;                       // in front of the first sequence or behind the last
  const int len = cache_length(c, b, status), kvh = h / (heads / c.kv);
  const int3 see = seen(mask, len - (r.y - row), len);
  for (int d = tid; d < c.dim; d += CS_THREADS) qs[d] = load1(q + row * q_stride + (long long)h * c.dim + d) * scale_log2;
  __syncthreads();
  float m = -CUDART_INF_F, l = 0.f, acc0 = 0.f, acc1 = 0.f;
  const int n = see.x + (see.z - see.y);
  for (int t0 = 0; t0 < n; t0 += CS_THREADS) {
    const int t = t0 + tid, j = t < see.x ? t : t - see.x + see.y;
    float s = -CUDART_INF_F, sv = 0.f;
    if (t < n) {
      s = simt_score(c, b, kvh, j, qs, status);
      const size_t at = (size_t)cache_page(c, b, j >> c.log_page, 0, status) * c.kv + kvh;
      sv = c.vs[at];
      vs_at[tid] = c.v + ((at << c.log_page) + (j & (c.page - 1))) * c.dim;
    }
    float mx = s;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, o));
    if ((tid & 31) == 0) red[tid >> 5] = mx;
    __syncthreads();
    const float m_new = fmaxf(m, fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
    const float base = m_new == -CUDART_INF_F ? 0.f : m_new, corr = exp2f(m - base);
    const float p = exp2f(s - base);
    ps[tid] = p * sv;
    l = l * corr + p;
    acc0 *= corr; acc1 *= corr;
    m = m_new;
    __syncthreads();
    const int cnt = min(CS_THREADS, n - t0);
    for (int i = 0; i < cnt; ++i) {
      const float w = ps[i];
      const uint8_t* v = vs_at[i];
      if (tid < c.dim) acc0 = fmaf(w, from_e4m3x2(v[tid]).x, acc0);
      if (tid + CS_THREADS < c.dim) acc1 = fmaf(w, from_e4m3x2(v[tid + CS_THREADS]).x, acc1);
    }
    __syncthreads();
  }
  l = warp_sum(l);
  __syncthreads();
  if ((tid & 31) == 0) red[tid >> 5] = l;
  __syncthreads();
  l = (red[0] + red[1]) + (red[2] + red[3]);
  const float inv = n > 0 ? 1.0f / l : 0.f;
  T* o = out + ((long long)row * heads + h) * c.dim;
  if (tid < c.dim) store1(o + tid, acc0 * inv);
  if (tid + CS_THREADS < c.dim) store1(o + tid + CS_THREADS, acc1 * inv);
  if (lse != nullptr && tid == 0)
    lse[(long long)row * heads + h] = n > 0 ? (m + log2f(l)) * 0.69314718055994531f : -CUDART_INF_F;
}

// One CTA per (text row, head) and sequence: weights of `count` tokens from `first` on.
template <class T>
__global__ void __launch_bounds__(CS_THREADS) k_cache_weights_simt(const CacheView c, const T* __restrict__ q,
                                                                  const int* __restrict__ cu, const float* __restrict__ lse,
                                                                  float* __restrict__ weights, long long q_stride,
                                                                  float scale_log2, int rows, int heads, const MaskRule mask,
                                                                  int n_text, int first, int count,
                                                                  unsigned* __restrict__ status) {
  __shared__ __align__(16) float qs[256];
  grid_dep_wait();
  grid_dep_launch();
  const int m = blockIdx.x % n_text, b = blockIdx.x / n_text, h = blockIdx.y, tid = threadIdx.x;
  const int2 r = cache_rows(cu, b, rows, status);
  const int row = r.y - n_text + m;
  float* o = weights + (((long long)b * heads + h) * n_text + m) * count;
  if (row < r.x) {
    for (int i = tid; i < count; i += CS_THREADS) o[i] = 0.f;
    return;
  }
  const int len = cache_length(c, b, status), kvh = h / (heads / c.kv);
  const int3 see = seen(mask, len - (r.y - row), len);
  for (int d = tid; d < c.dim; d += CS_THREADS) qs[d] = load1(q + row * q_stride + (long long)h * c.dim + d) * scale_log2;
  __syncthreads();
  const float base = lse[(long long)row * heads + h] * 1.4426950408889634f;
  for (int i = tid; i < count; i += CS_THREADS) {
    const long long j = (long long)first + i;
    const bool on = j < see.x || (j >= see.y && j < see.z);
    o[i] = on ? exp2f(simt_score(c, b, kvh, (int)j, qs, status) - base) : 0.f;
  }
}

}  // namespace ficoco
