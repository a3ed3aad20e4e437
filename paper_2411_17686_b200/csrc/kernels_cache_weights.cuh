// Attention weights of the last rows of every sequence over a range of its tokens (what ficoco_l_reduce takes), on the tensor cores.
//
// S^T = K Q^T: the keys' codes are operand A (128 tokens), RC query rows with NT e4m3 terms each are the columns, so that a
// thread has one token and a warp writes 32 neighbours of a row of the result at once.  weight = 2^(log2 score - log2 of the
// row's denominator), which the attention call before it has left in lse.
//
// What bounds it: writing the result, 4 bytes per weight, against 1 byte of key for RC of them.  A CTA owns RC rows of one head
// group and a run of tiles of tokens; the host sizes the runs so that every SM has some.
// Roles: warps 0-3 queries and output, warp 4 TMA, warp 5 MMA.
#pragma once
#include "cache_umma.cuh"

namespace ficoco {

constexpr int WEIGHT_THREADS = 192;

template <int DIM, int NT, int RC>
struct WeightPlan {
  static constexpr int N = NT * RC, KEYS = CTILE * DIM, STAGES = 3;
  static constexpr int Q_BYTES = (N * DIM + 1023) / 1024 * 1024;
  static constexpr int SMEM = 1024 + STAGES * KEYS + Q_BYTES;
  static constexpr int TMEM = 2 * N <= 128 ? 128 : 256;
  static constexpr int PER_SM = TMEM == 128 ? 4 : 2;
  static_assert(2 * N <= 256 && N % 16 == 0 && RC % 16 == 0, "two CTAs per SM");
};

template <class T, int DIM, int NT, int RC>
__global__ void __launch_bounds__(WEIGHT_THREADS, (WeightPlan<DIM, NT, RC>::PER_SM)) k_cache_weights(
    const __grid_constant__ CUtensorMap kmap, const CacheView c, const T* __restrict__ q, const int* __restrict__ cu,
    const float* __restrict__ lse, float* __restrict__ weights, long long q_stride, float scale_log2, int rows, int heads,
    const MaskRule mask, int n_text, int first, int count, int tiles_per_cta, unsigned* __restrict__ status,
    unsigned long long wait_ns) {
  using PL = WeightPlan<DIM, NT, RC>;
  constexpr int N = PL::N, NST = PL::STAGES;
  extern __shared__ unsigned char weight_raw[];
  __shared__ uint64_t k_full[NST], k_empty[NST], q_bar, s_bar[2], s_free[2], drain_bar;
  __shared__ uint32_t tmem_s;
  __shared__ int dead_s;
  __shared__ float q_scale[RC];
  __shared__ __align__(16) uint4 row_is[RC];           // scale of the row's scores, log2 of its denominator, where its weights lie
  __shared__ int4 row_see[RC];                         // tokens [0, x) and [y, z)
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t k_ring = (smem_u32(weight_raw) + 1023u) & ~1023u, q_base = k_ring + NST * PL::KEYS;
  const int group = heads / c.kv;
  if (tid == 0) {
    for (int s = 0; s < NST; ++s) { mbar_init(&k_full[s], 1); mbar_init(&k_empty[s], 1); }
    mbar_init(&q_bar, 4);
    for (int s = 0; s < 2; ++s) { mbar_init(&s_bar[s], 1); mbar_init(&s_free[s], 4); }
    mbar_init(&drain_bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 5) tmem_alloc(&tmem_s, PL::TMEM);
  grid_dep_wait();
  if (tid == 0) dead_s = (*reinterpret_cast<const volatile unsigned*>(status) & STATUS_TIMEOUT) ? 1 : 0;
  const int head = blockIdx.y % c.kv, b = blockIdx.y / c.kv, x0 = blockIdx.z * RC, tile0 = first / CTILE + blockIdx.x * tiles_per_cta;
  const int tiles = min(tiles_per_cta, (first + count + CTILE - 1) / CTILE - tile0);
  const int2 r = cache_rows(cu, b, rows, status);
  const int len = cache_length(c, b, status);
  ctc_fence_before();
  __syncthreads();
  ctc_fence_after();
  grid_dep_launch();       // behind the barrier: a dependent that took this SM's TMEM first would wait for it for ever
  const uint32_t tmem = tmem_s;
  bool ok = !dead_s;                                   // the same in all lanes of a warp
  auto wait = [&](uint64_t* bar, int phase) { ok = ok && __all_sync(0xFFFFFFFFu, mbar_wait(bar, (uint32_t)phase & 1u, wait_ns)); };
  const bool dead = !ok;

  if (warp == 4) {
    // ---------------- TMA: lane p brings page p of a tile ----------------------------------------------------------------
    const uint32_t bytes = (uint32_t)(c.page * DIM);
    auto page_of = [&](int k) {
      const int at = k < tiles ? (tile0 + k) * CTILE + (lane << c.log_page) : len;
      return lane < (CTILE >> c.log_page) && at < len ? cache_page(c, b, at >> c.log_page, 0, status) : -1;
    };
    int page = page_of(0), i = 0;
    for (; ok && i < tiles; ++i) {
      const int next = page_of(i + 1), st = i % NST;
      const uint32_t load = bytes * (uint32_t)__popc(__ballot_sync(0xFFFFFFFFu, page >= 0));
      if (i >= NST) wait(&k_empty[st], i / NST - 1);
      if (!ok) break;
      if (lane == 0) mbar_expect_tx(&k_full[st], load);
      __syncwarp();
      if (page >= 0) tma_rows(k_ring + st * PL::KEYS + lane * bytes, &kmap, (page * c.kv + head) << c.log_page, &k_full[st]);
      page = next;
    }
    if (!ok && !dead) {
      if (lane == 0) atomicOr(status, STATUS_TIMEOUT);
      for (int k = max(0, i - NST); k < i; ++k) mbar_wait(&k_full[k % NST], (k / NST) & 1, wait_ns);
    }
  } else if (warp == 5) {
    // ---------------- MMA ------------------------------------------------------------------------------------------------
    const uint32_t u_tmem = __shfl_sync(0xFFFFFFFFu, tmem, 0);
    constexpr uint32_t idesc = cache_idesc(128, N, 0, 0);
    const uint64_t bd = cache_desc<DIM>(q_base);
    wait(&q_bar, 0);
    for (int i = 0; ok && i < tiles; ++i) {
      wait(&k_full[i % NST], i / NST);
      if (i >= 2) wait(&s_free[i & 1], (i >> 1) - 1);
      if (!ok) break;
      ctc_fence_after();
      const uint64_t ad = cache_desc<DIM>(k_ring + (uint32_t)(i % NST) * PL::KEYS);
#pragma unroll
      for (int k = 0; k < DIM / 32; ++k) mma_f8(u_tmem + (uint32_t)(i & 1) * N, ad + 2 * k, bd + 2 * k, idesc, k > 0);
      mma_commit(&s_bar[i & 1]);
      mma_commit(&k_empty[i % NST]);
    }
    if (!ok && !dead) {
      if (lane == 0) atomicOr(status, STATUS_TIMEOUT);
      mma_commit(&drain_bar);
      mbar_wait(&drain_bar, 0, wait_ns);
    }
  } else if (!dead) {
    // ---------------- queries, then output: thread = token -----------------------------------------------------------------
    // row x of the chunk: text row x / group of the last n_text, head x % group of the group
    const int n_rows = r.y - r.x;
    auto row_of = [&](int x, int& h) {                 // row of q, -1 where the sequence has none
      const int m = x / group;
      h = head * group + x - m * group;
      const int i = n_rows - n_text + m;
      return m < n_text && i >= 0 ? r.x + i : -1;
    };
    constexpr int LANES = DIM / 8, AT_ONCE = 128 / LANES, PASSES = (RC + AT_ONCE - 1) / AT_ONCE;
    const int chunk = tid % LANES;
    Raw8<T> raw[PASSES];                               // all in flight at once (one after the other: 8 us for 64 rows)
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      int h;
      const int row = row_of(x0 + p * AT_ONCE + tid / LANES, h);
      if (row >= 0) raw[p].load(q + (long long)row * q_stride + (long long)h * DIM + chunk * 8);
      else raw[p].clear();
    }
    float scale[PASSES];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      float f[8];
      raw[p].get(f);
      scale[p] = query_scale<DIM>(f);
    }
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int x = p * AT_ONCE + tid / LANES;
      float f[8];
      raw[p].get(f);
      if (x < RC) {
        store_query<DIM, NT>(f, scale[p], q_base, x, RC, chunk);
        if (chunk == 0) q_scale[x] = scale[p] * scale_log2;
      }
    }
    int in_lo = 0, in_hi = INT32_MAX;                  // tokens that all rows of the chunk see
    for (int x = tid; x < RC; x += 128) {
      int h;
      const int row = row_of(x0 + x, h), m = (x0 + x) / group;
      const int3 see = seen(mask, len - (r.y - row), len);
      row_see[x] = row >= 0 ? make_int4(see.x, see.y, see.z, 0) : make_int4(0, 0, 0, 0);
      const float base = row >= 0 ? lse[(long long)row * heads + h] * 1.4426950408889634f : 0.f;
      row_is[x] = make_uint4(0u, __float_as_uint(base), (uint32_t)((h - head * group) * n_text + m) * (uint32_t)count, 0u);
    }
    fence_proxy_async();
    __syncwarp();
    if (lane == 0) mbar_arrive(&q_bar);
    cta_sync(1, 128);
    if (tid < RC) row_is[tid].x = __float_as_uint(q_scale[tid]);
    cta_sync(1, 128);
    float* const to = weights + ((long long)b * heads + head * group) * n_text * count - first;
    const int n_x = min(RC, n_text * group - x0);
    in_lo = row_see[n_x - 1].y;
    in_hi = row_see[0].z;                              // (rows in order of position: the first sees least ahead, the last least behind)
    const uint32_t t_lane = tmem + ((uint32_t)(warp * 32) << 16);
    for (int i = 0; i < tiles; ++i) {
      const int base = (tile0 + i) * CTILE, j = base + tid;
      const int pg = j < len ? cache_page(c, b, j >> c.log_page, 0, status) : 0;
      const float ks = j < len ? c.ks[(size_t)pg * c.kv + head] : 0.f;
      wait(&s_bar[i & 1], i >> 1);
      if (!ok) break;
      ctc_fence_after();
      const bool edge = base < in_lo || base + CTILE > in_hi, mine = j >= first && j < first + count;
#pragma unroll 1
      for (int x = 0; x < n_x; x += 16) {
        float s[16];
#pragma unroll
        for (int u = NT - 1; u >= 0; --u) {
          float f[16];
          ctmem_ld16(t_lane + (uint32_t)(i & 1) * N + u * RC + x, f);
          ctmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 16; ++e) s[e] = u == NT - 1 ? f[e] : fmaf(s[e], 0.0625f, f[e]);
        }
        uint32_t at[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const uint4 is = row_is[x + e];
          s[e] = ex2(fmaf(s[e], __uint_as_float(is.x) * ks, -__uint_as_float(is.y)));
          at[e] = is.z + (uint32_t)j;
        }
        if (edge) {
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int4 see = row_see[x + e];
            s[e] = j < see.z && (j >= see.y || j < see.x) ? s[e] : 0.f;
          }
        }
        if (mine) {
          if (x + 16 <= n_x) {
#pragma unroll
            for (int e = 0; e < 16; ++e) to[at[e]] = s[e];
          } else {
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (x + e < n_x) to[at[e]] = s[e];
          }
        }
      }
      ctc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&s_free[i & 1]);
    }
    if (!ok && lane == 0) atomicOr(status, STATUS_TIMEOUT);
  }
  ctc_fence_before();
  __syncthreads();
  if (warp == 5) tmem_free(tmem, PL::TMEM);
}

}  // namespace ficoco
