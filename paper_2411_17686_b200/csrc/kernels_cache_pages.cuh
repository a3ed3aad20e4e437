// Kernels that write pages of the 8-bit cache: append, compact, copy.
//
// Append and compact share one shape.  A CTA owns one page and some of its key/value heads; a team of threads (a power of two,
// a warp at least, sized by the host so that its part of the page stays in registers) works on the keys or the values of one head.
// It reads its rows once for the largest magnitude, settles the scale (a power of two, so that the division is exact and the only
// rounding is the one to e4m3) and converts what it holds.  Which sequence a CTA belongs to follows from cu_rows and the
// lengths on the device; the host sizes the grid for the most pages that so many rows can touch (rows / page + 2 per sequence), the
// CTAs beyond return at once.
// What bounds them: instruction issue and HBM on prompts, the chain of lookups (sequence, length, page, old scale) on single tokens.
// Measured, replayed from a graph: append of 16 prompts of 640 rows, 32 heads of 128, bf16, 55 us, 4.5 TB/s, fp32 76 us; one row of 64 sequences
// 4.2 us (6.9 called from Python one after the other, which is the host's time); compact of 48 sequences in pages of 16, 32 heads, 151 us, 4.1
// TB/s; copy of 190 pages of 128 tokens and 8 heads 20.6 us, 4.8 TB/s (17.8 called one after the other on one pool, whose pages stay in L2).
#pragma once
#include "cache_common.cuh"

namespace ficoco {

constexpr int PAGE_LOG = 8, PAGE_THREADS = 1 << PAGE_LOG;
// Vectors that a thread keeps between the two passes; more are read again.  As much as the registers take without spilling, four CTAs
// per SM (three for compact): 16 prompts of 640 rows and 32 heads 53 us with eight, 78 with four; single tokens of 64 sequences 6.2 us
// with eight (most of them empty), 4.3 with four; 48 gathered sequences 153 us with four and three CTAs, 172 with four CTAs, 211 with
// three vectors.
constexpr int APPEND_HELD = 8, STEP_HELD = 4, COMPACT_HELD = 4;

// Largest of `v` over the team of this thread (all values >= 0).
__device__ __forceinline__ float team_max(float v, int team_warps, float (&warp_max)[PAGE_THREADS / 32]) {
  const int warp = threadIdx.x >> 5;
  v = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(v)));
  if (team_warps == 1) return v;
  __syncthreads();                        // (what an earlier call left has been read)
  if ((threadIdx.x & 31) == 0) warp_max[warp] = v;
  __syncthreads();
  const int w0 = warp & ~(team_warps - 1);
  v = warp_max[w0];
  for (int w = 1; w < team_warps; ++w) v = fmaxf(v, warp_max[w0 + w]);
  return v;
}

// The largest magnitude of many vectors, as an integer (infinity and NaN are the largest): bits of fp32, or the bits of bf16 in both
// halves of a word, two to an instruction.
__device__ __forceinline__ uint32_t top_of(uint32_t top, const Raw8<float>& r) {
  const float f[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
#pragma unroll
  for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(f[j]) & 0x7FFFFFFFu);
  return top;
}
__device__ __forceinline__ uint32_t top_of(uint32_t top, const Raw8<__nv_bfloat16>& r) {
  constexpr uint32_t ABS = 0x7FFF7FFFu;
  return __vimax3_u16x2(__vimax3_u16x2(top, r.a.x & ABS, r.a.y & ABS), r.a.z & ABS, r.a.w & ABS);
}
__device__ __forceinline__ uint32_t top_bits(uint32_t top, const float*) { return top; }                       // as bits of fp32
__device__ __forceinline__ uint32_t top_bits(uint32_t top, const __nv_bfloat16*) { return max(top & 0xFFFFu, top >> 16) << 16; }

template <class T, int HELD>
__global__ void __launch_bounds__(PAGE_THREADS, (sizeof(T) == 2 || HELD == STEP_HELD ? 4 : 2)) k_cache_append(const CacheView c, const T* __restrict__ k, const T* __restrict__ v,
                                                              const int* __restrict__ cu, long long k_stride, long long v_stride,
                                                              int rows, int log_team, unsigned* __restrict__ status) {
  __shared__ float warp_max[PAGE_THREADS / 32];
  __shared__ unsigned poisoned[PAGE_THREADS / 64][4];          // per head of the CTA: rows of the page that hold a NaN or an infinity
  grid_dep_wait();
  grid_dep_launch();
  const int u = blockIdx.x, tid = threadIdx.x;
  if (tid < PAGE_THREADS / 64 * 4) poisoned[tid >> 2][tid & 3] = 0u;
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

  const int team = 1 << log_team, mine = tid >> log_team, lane = tid & (team - 1);
  const int pair = (blockIdx.y << (PAGE_LOG - log_team)) + mine, head = pair >> 1;       // (head, keys or values); two teams of a head side by side
  const bool is_v = pair & 1, on = head < c.kv;
  const int vecs = c.dim >> 3, total = on ? (s1 - s0) * vecs : 0;                 // vectors of eight elements
  const long long stride = is_v ? v_stride : k_stride;
  const T* src = (is_v ? v : k) + (long long)row0 * stride + (on ? head : 0) * c.dim;
  const size_t at = (size_t)page * c.kv + (on ? head : 0);
  uint8_t* dst = (is_v ? c.v : c.k) + (at << c.log_page) * c.dim;
  float* scale = (is_v ? c.vs : c.ks) + at;
  const float old = s0 > 0 ? *scale : 0.f;
  const uint32_t inv_vecs = ((1u << 20) + vecs - 1) / vecs;     // i / vecs as a product: exact for i < 2^20 / vecs, a page has 2^12
  auto row_of = [&](int i) { return (int)((uint32_t)i * inv_vecs >> 20); };
  auto from_row = [&](int i, int row) { return src + row * stride + (i - row * vecs) * 8; };

  Raw8<T> held[HELD];
#pragma unroll
  for (int x = 0; x < HELD; ++x) {
    const int i = lane + (x << log_team);
    if (i < total) held[x].load(from_row(i, row_of(i)));
    else held[x].clear();
  }
  uint32_t top = 0;
#pragma unroll
  for (int x = 0; x < HELD; ++x) top = top_of(top, held[x]);
#pragma unroll 1
  for (int i = lane + (HELD << log_team); i < total; i += team) {
    Raw8<T> raw;
    raw.load(from_row(i, row_of(i)));
    top = top_of(top, raw);
  }
  top = top_bits(top, k);
  const bool any_bad = __syncthreads_or(top >= 0x7F800000u);
  auto is_bad = [&](int row) { return (poisoned[mine >> 1][row >> 5] >> (row & 31) & 1u) != 0; };
  if (any_bad) {                          // rare: which rows, then once more without them
#pragma unroll 1
    for (int i = lane; i < total; i += team) {
      const int row = row_of(i);
      Raw8<T> raw;
      raw.load(from_row(i, row));
      if (top_bits(top_of(0, raw), k) >= 0x7F800000u) atomicOr(&poisoned[mine >> 1][row >> 5], 1u << (row & 31));
    }
    __syncthreads();
    top = 0;
#pragma unroll 1
    for (int i = lane; i < total; i += team) {
      const int row = row_of(i);
      Raw8<T> raw;
      raw.load(from_row(i, row));
      if (!is_bad(row)) top = max(top, top_bits(top_of(0, raw), k));
    }
  }
  const float amax = team_max(__uint_as_float(top), team >> 5, warp_max);
  if (!on) return;
  const float s = fmaxf(scale_of(amax), old), inv = 1.0f / s;
  if (s0 > 0 && s > old) {                // the older codes of the page move to the larger scale
    const float f = old * inv;
#pragma unroll 1
    for (int i = lane; i < s0 * vecs; i += team) {
      uint2* p = reinterpret_cast<uint2*>(dst) + i;
      float x[8];
      from_e4m3x8(*p, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] *= f;
      *p = to_e4m3x8(x);
    }
  }
  uint2* out = reinterpret_cast<uint2*>(dst) + s0 * vecs;
  auto put = [&](const Raw8<T>& raw, int i) {
    float f[8];
    raw.get(f);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] *= inv;
    uint2 codes = to_e4m3x8(f);
    if (any_bad && is_bad(row_of(i))) codes = is_v ? make_uint2(0u, 0u) : make_uint2(E4M3_NAN4, E4M3_NAN4);
    out[i] = codes;
  };
#pragma unroll
  for (int x = 0; x < HELD; ++x) {
    const int i = lane + (x << log_team);
    if (i < total) put(held[x], i);
  }
#pragma unroll 1
  for (int i = lane + (HELD << log_team); i < total; i += team) {
    Raw8<T> raw;
    raw.load(from_row(i, row_of(i)));
    put(raw, i);
  }
  if (lane == 0) *scale = s;
}

__global__ void __launch_bounds__(PAGE_THREADS, 3) k_cache_compact(const CacheView c, const int* __restrict__ to_table,
                                                               const int* __restrict__ kept, const int* __restrict__ cu,
                                                               int* __restrict__ lengths_out, long long to_stride,
                                                               int to_pages, int n_kept, int first, int log_team,
                                                               unsigned* __restrict__ status) {
  __shared__ float warp_max[PAGE_THREADS / 32];
  __shared__ int2 row_from[128];                               // page and slot of each row of the new page
  grid_dep_wait();
  grid_dep_launch();
  const int u = blockIdx.x, tid = threadIdx.x;
  auto unit0 = [&](int s) { return ((max(cu[s], 0) + (long long)s * first) >> c.log_page) + 2 * s; };
  const int b = owner_of(c.batch, unit0, u);
  const int2 r = cache_rows(cu, b, n_kept, status);
  const int len = cache_length(c, b, status), front = min(first, len), total_rows = front + (r.y - r.x);
  const int pi = (int)(u - unit0(b));
  if (pi == 0 && blockIdx.y == 0 && tid == 0 && lengths_out != nullptr) lengths_out[b] = total_rows;
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
      const bool inside = e >= 0 && e < len - front;             // (front + e alone can pass 32 bits)
      if (!inside) atomicOr(status, STATUS_CACHE);
      pos = inside ? front + e : 0;
    }
    // a sequence without tokens has nothing to gather, not even token 0: zeros (page -1)
    row_from[tid] = make_int2(len > 0 ? cache_page(c, b, pos >> c.log_page, 0, status) : -1, pos & (c.page - 1));
  }
  __syncthreads();
  const int team = 1 << log_team, mine = tid >> log_team, lane = tid & (team - 1);
  const int groups = ((2 * c.kv << log_team) + PAGE_THREADS - 1) >> PAGE_LOG;
  // one look-up of the page and its rows for as many heads as the grid leaves to a CTA
#pragma unroll 1
  for (int part = blockIdx.y; part < groups; part += gridDim.y) {
    const int pair = (part << (PAGE_LOG - log_team)) + mine, head = pair >> 1;
    const bool is_v = pair & 1, on = head < c.kv;
    const int vecs = c.dim >> 4, total = on ? s1 * vecs : 0;      // vectors of 16 codes
    const uint8_t* src = is_v ? c.v : c.k;
    const float* scales = is_v ? c.vs : c.ks;
    const uint32_t inv_vecs = ((1u << 20) + vecs - 1) / vecs;     // i / vecs as a product: exact for i < 2^20 / vecs, a page has 2^11
    auto fetch = [&](int i, uint4& codes, float& s) {
      const int row = (int)((uint32_t)i * inv_vecs >> 20);
      const int2 f = row_from[row];
      const size_t at = (size_t)max(f.x, 0) * c.kv + head;
      codes = *reinterpret_cast<const uint4*>(src + ((at << c.log_page) + f.y) * c.dim + (i - row * vecs) * 16);
      s = f.x >= 0 ? scales[at] : 0.f;
    };
    auto look = [&](const uint4& u4, float s) {
      const uint32_t w[4] = {u4.x, u4.y, u4.z, u4.w};
      float m = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float2 a = from_e4m3x2(w[k] & 0xFFFFu), d = from_e4m3x2(w[k] >> 16);
        m = fmaxf(fmaxf(m, fmaxf(fabsf(a.x), fabsf(a.y))), fmaxf(fabsf(d.x), fabsf(d.y)));       // (a NaN key counts for nothing)
      }
      return m * s;
    };
    uint4 held[COMPACT_HELD];
    float hs[COMPACT_HELD];
#pragma unroll
    for (int x = 0; x < COMPACT_HELD; ++x) {
      const int i = lane + (x << log_team);
      held[x] = make_uint4(0u, 0u, 0u, 0u);
      hs[x] = 0.f;
      if (i < total) fetch(i, held[x], hs[x]);
    }
    float amax = 0.f;
#pragma unroll
    for (int x = 0; x < COMPACT_HELD; ++x) amax = fmaxf(amax, look(held[x], hs[x]));
#pragma unroll 1
    for (int i = lane + (COMPACT_HELD << log_team); i < total; i += team) {
      uint4 u4;
      float s;
      fetch(i, u4, s);
      amax = fmaxf(amax, look(u4, s));
    }
    amax = team_max(amax, team >> 5, warp_max);
    if (!on) continue;                                            // (whole teams; the barriers in between are reached by all)
    const size_t at = (size_t)page * c.kv + head;
    const float s = scale_of(amax), inv2 = 2.0f / s;
    uint4* out = reinterpret_cast<uint4*>((is_v ? c.v : c.k) + (at << c.log_page) * c.dim);
    auto put = [&](int i, const uint4& u4, float by) {
      const uint32_t w[4] = {u4.x, u4.y, u4.z, u4.w};
      const float half = 0.5f * by;
      uint32_t o[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {          // exact: powers of two (their quotient alone can overflow, a value itself be 2^128 and more)
        const float2 a = from_e4m3x2(w[k] & 0xFFFFu), d = from_e4m3x2(w[k] >> 16);
        o[k] = to_e4m3x2(a.x * half * inv2, a.y * half * inv2) | to_e4m3x2(d.x * half * inv2, d.y * half * inv2) << 16;
      }
      out[i] = make_uint4(o[0], o[1], o[2], o[3]);
    };
#pragma unroll
    for (int x = 0; x < COMPACT_HELD; ++x) {
      const int i = lane + (x << log_team);
      if (i < total) put(i, held[x], hs[x]);
    }
#pragma unroll 1
    for (int i = lane + (COMPACT_HELD << log_team); i < total; i += team) {
      uint4 u4;
      float by;
      fetch(i, u4, by);
      put(i, u4, by);
    }
    if (lane == 0) (is_v ? c.vs : c.ks)[at] = s;
  }
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
