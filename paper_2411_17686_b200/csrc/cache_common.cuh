// Shared device code of the 8-bit paged cache: the view of a cache, checked lookups, e4m3 conversions, the scale rule.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math_constants.h>
#include <stdint.h>
#include "async_ops.cuh"
#include "common.cuh"

namespace ficoco {

constexpr unsigned STATUS_CACHE = 16u;    // a page, length, row offset or kept index was out of range

struct CacheView {
  uint8_t* k;
  uint8_t* v;
  float* ks;
  float* vs;
  const int* table;
  const int* len;
  long long table_stride;
  int n_pages, page, log_page, kv, dim, batch, max_pages;
};

// Tokens of sequence b, cut to what its table can hold.
__device__ __forceinline__ int cache_length(const CacheView& c, int b, unsigned* status) {
  const int n = c.len[b], cap = (int)min((long long)c.max_pages << c.log_page, (long long)INT32_MAX);
  if ((unsigned)n <= (unsigned)cap) return n;
  atomicOr(status, STATUS_CACHE);
  return n < 0 ? 0 : cap;
}
// Page of entry i of b's table; one outside the pool becomes `instead`.
__device__ __forceinline__ int cache_page(const CacheView& c, int b, int i, int instead, unsigned* status) {
  const int p = c.table[(long long)b * c.table_stride + i];
  if ((unsigned)p < (unsigned)c.n_pages) return p;
  atomicOr(status, STATUS_CACHE);
  return instead;
}
// Rows [lo, hi) of sequence b, cut to the rows of the call.
__device__ __forceinline__ int2 cache_rows(const int* cu, int b, int rows, unsigned* status) {
  const int lo = cu[b], hi = cu[b + 1];
  if (lo >= 0 && hi >= lo && hi <= rows) return make_int2(lo, hi);
  atomicOr(status, STATUS_CACHE);
  const int l = min(max(lo, 0), rows);
  return make_int2(l, max(l, min(hi, rows)));
}
// Sequence of the call that owns unit u, where sequence b owns the units from first(b) on and first is not
// decreasing: the number of b in [1, batch) with first(b) <= u.  The whole CTA takes part (one trip to memory for up to
// blockDim.x sequences, where a binary search takes one per halving).
template <class F>
__device__ __forceinline__ int owner_of(int batch, F first, long long u) {
  int below = 0;
  for (int b0 = 1; b0 < batch; b0 += blockDim.x) {
    const int b = b0 + threadIdx.x;
    const int n = __syncthreads_count(b < batch && first(b) <= u);
    below += n;
    if (n < (int)blockDim.x) break;
  }
  return below;
}

// The smallest power of two >= 2^-64 that brings amax to 448 = 1.75 * 2^8 or below.
__device__ __forceinline__ float scale_of(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return __uint_as_float((uint32_t)(max(e, -64) + 127) << 23);
}

// Two values to two e4m3 codes (lo in the low byte), nearest even, beyond 448 to 448; NaN stays NaN.
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {
  uint16_t d;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(d) : "f"(hi), "f"(lo));
  return d;
}
__device__ __forceinline__ float2 from_e4m3x2(uint32_t codes) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)codes));
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
// Eight codes.
__device__ __forceinline__ void from_e4m3x8(const uint2& u, float (&f)[8]) {
  const float2 a = from_e4m3x2(u.x & 0xFFFFu), b = from_e4m3x2(u.x >> 16);
  const float2 c = from_e4m3x2(u.y & 0xFFFFu), d = from_e4m3x2(u.y >> 16);
  f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y; f[4] = c.x; f[5] = c.y; f[6] = d.x; f[7] = d.y;
}
__device__ __forceinline__ uint2 to_e4m3x8(const float (&f)[8]) {
  return make_uint2(to_e4m3x2(f[0], f[1]) | to_e4m3x2(f[2], f[3]) << 16, to_e4m3x2(f[4], f[5]) | to_e4m3x2(f[6], f[7]) << 16);
}
constexpr uint32_t E4M3_NAN4 = 0x7F7F7F7Fu;

// Eight consecutive elements of a row as they lie in memory, for loads that are to be in flight together.
template <class T> struct Raw8;
template <> struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = *reinterpret_cast<const float4*>(p); b = *reinterpret_cast<const float4*>(p + 4); }
  __device__ __forceinline__ void clear() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
};
template <> struct Raw8<__nv_bfloat16> {
  uint4 a;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { a = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void clear() { a = make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ void get(float (&f)[8]) const { unpack(a, f, (const __nv_bfloat16*)nullptr); }
};
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store1(float* p, float x) { *p = x; }
__device__ __forceinline__ void store1(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }
__device__ __forceinline__ void store4(float* p, const float4& v) { *reinterpret_cast<float4*>(p) = v; }
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float4& v) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
}

// What the rows of a call see.
struct MaskRule {
  int window, sinks, causal;
};
// Tokens [0, sinks_hi) and [lo, hi) seen by the row at position pos of a sequence of len tokens (sinks_hi <= lo).
__device__ __forceinline__ int3 seen(const MaskRule& m, int pos, int len) {
  const int hi = m.causal ? max(0, min(len, pos + 1)) : len;
  const int lo = m.window > 0 ? min(max(0, pos - m.window + 1), hi) : 0;
  return make_int3(min(m.sinks, lo), lo, hi);
}

}  // namespace ficoco
