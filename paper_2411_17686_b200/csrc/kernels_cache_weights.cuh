// Attention weights of the last rows of every sequence over a range of its tokens (what ficoco_l_reduce takes), on the tensor cores.
//
// S^T = K Q^T: the keys' codes are operand A (128 tokens), RC query rows with NT e4m3 terms each are the columns, so that a
// thread has one token and a warp writes 32 neighbours of a row of the result at once.  weight = 2^(log2 score - log2 of the
// row's denominator), which the attention call before it has left in lse.
//
// What bounds it: writing the result, 4 bytes per weight, against 1 byte of key for RC of them.  The tiles of all (sequence, head,
// chunk of RC rows) items form one list which is cut into equal pieces, one per CTA, two CTAs per SM; the next item's query rows
// are fetched and split by warps of their own while this one's weights are written (one item per CTA, its rows fetched first,
// left the memory idle a third of the time: 39 us for 16 sequences of 64 x 576 weights and 32 heads).
// Roles: warps 0-3 and 4-7 output, every other tile each (thread = token), warps 8-11 queries, warp 12 TMA and key scales, warp 13
// MMA.
//
// Measured: 16 sequences, 64 text rows over 576 tokens, 32 heads, bf16 (75 MB of results, 38 MB of keys): 36 us; the stores alone 16.5.  One
// sequence of 37 over 2880, fp32, 32 heads on 8: 14.4 us.
#pragma once
#include "cache_umma.cuh"

namespace ficoco {

constexpr int WEIGHT_THREADS = 448;

template <int DIM, int NT, int RC>
struct WeightPlan {
  static constexpr int N = NT * RC, KEYS = CTILE * DIM, STAGES = 3, SCALES = 8;
  static constexpr int Q_BYTES = (N * DIM + 1023) / 1024 * 1024;
  static constexpr int SMEM = 1024 + STAGES * KEYS + 2 * Q_BYTES;
  static constexpr int TMEM = 2 * N <= 128 ? 128 : 256;
  static_assert(2 * N <= 256 && N % 16 == 0 && RC % 16 == 0 && SMEM <= 104 * 1024, "two CTAs per SM");
  static_assert(SCALES >= STAGES + 2, "a tile's scales outlive its keys by the two score buffers");
};

template <class T, int DIM, int NT, int RC>
__global__ void __launch_bounds__(WEIGHT_THREADS, 2) k_cache_weights(
    const __grid_constant__ CUtensorMap kmap, const CacheView c, const T* __restrict__ q, const int* __restrict__ cu,
    const float* __restrict__ lse, float* __restrict__ weights, long long q_stride, float scale_log2, int rows, int heads,
    const MaskRule mask, int n_text, int first, int count, int tiles, int chunks, unsigned* __restrict__ status,
    unsigned long long wait_ns, int extra_arrivals) {
  using PL = WeightPlan<DIM, NT, RC>;
  constexpr int N = PL::N, NST = PL::STAGES, NSC = PL::SCALES;
  extern __shared__ unsigned char weight_raw[];
  __shared__ uint64_t k_full[NST], k_empty[NST], sc_bar[NSC], q_bar[2], q_free[2], s_bar[2], s_free[2], drain_bar;
  __shared__ uint32_t tmem_s;
  __shared__ int dead_s;
  __shared__ float key_scale[NSC][8];
  __shared__ __align__(16) float row_is[2][RC / 2][4]; // of a pair of rows: the scales of their scores, minus log2 of their denominators
  __shared__ int4 row_see[2][RC];                      // tokens [0, x) and [y, z)
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t k_ring = (smem_u32(weight_raw) + 1023u) & ~1023u, q_base = k_ring + NST * PL::KEYS;
  const int group = heads / c.kv;
  if (tid == 0) {
    for (int s = 0; s < NST; ++s) { mbar_init(&k_full[s], 1); mbar_init(&k_empty[s], 1); }
    for (int s = 0; s < NSC; ++s) mbar_init(&sc_bar[s], 1);
    for (int s = 0; s < 2; ++s) { mbar_init(&q_bar[s], 4 + extra_arrivals); mbar_init(&q_free[s], 8); mbar_init(&s_bar[s], 1); mbar_init(&s_free[s], 4); }
    mbar_init(&drain_bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 13) tmem_alloc(&tmem_s, PL::TMEM);
  grid_dep_wait();
  if (tid == 0) dead_s = (*reinterpret_cast<const volatile unsigned*>(status) & STATUS_TIMEOUT) ? 1 : 0;
  ctc_fence_before();
  __syncthreads();
  ctc_fence_after();
  grid_dep_launch();       // behind the barrier: a dependent that took this SM's TMEM first would wait for it for ever
  const uint32_t tmem = tmem_s;
  // ---- this CTA's piece of the list: tiles [piece0, piece1) of items (sequence, head, chunk), chunks innermost ----------------
  const long long total = (long long)c.batch * c.kv * chunks * tiles;
  const long long piece0 = total * blockIdx.x / gridDim.x, piece1 = dead_s ? piece0 : total * (blockIdx.x + 1) / gridDim.x;
  struct Seg { int b, head, chunk, tile, count; };
  const int item0 = (int)(piece0 / tiles);             // (the host keeps the number of items below 2^31)
  Seg at;
  at.chunk = item0 % chunks; at.head = item0 / chunks % c.kv; at.b = item0 / chunks / c.kv;
  at.tile = (int)(piece0 - (long long)item0 * tiles);
  long long left = piece1 - piece0;
  auto next = [&](Seg& g) {
    if (left <= 0) return false;
    g = at;
    g.count = (int)min((long long)(tiles - at.tile), left);
    left -= g.count;
    at.tile = 0;
    if (++at.chunk == chunks) {
      at.chunk = 0;
      if (++at.head == c.kv) { at.head = 0; ++at.b; }
    }
    return true;
  };
  bool ok = true;                                      // the same in all lanes of a warp
  auto wait = [&](uint64_t* bar, int phase) { ok = ok && warp_wait(bar, (uint32_t)phase & 1u, wait_ns); };
  // x / n_text as a product: ceil(2^32 / n_text), exact while x * n_text < 2^32 (the host sees to that); 1 gives 2^32 = 0
  const uint32_t inv_text = n_text == 1 ? 0u : 0xFFFFFFFFu / (uint32_t)n_text + 1u;
  // row x of a head group: text row x % n_text of the last n_text, head x / n_text of the group, so that its weights lie
  // x * count behind the group's first; -1 where the sequence has no such row
  auto row_of = [&](const Seg& g, const int2& r, int x, int& h, int& m) {
    const int e = inv_text == 0u ? x : (int)__umulhi((uint32_t)x, inv_text);
    m = x - e * n_text;
    h = g.head * group + e;
    const int i = r.y - r.x - n_text + m;
    return e < group && i >= 0 ? r.x + i : -1;
  };
  Seg g;

  if (warp == 12) {
    // ---------------- TMA: lane p brings page p of a tile ----------------------------------------------------------------
    const uint32_t bytes = (uint32_t)(c.page * DIM);
    int i = 0;
    while (ok && next(g)) {
      const int len = cache_length(c, g.b, status);
      auto page_of = [&](int t) {
        const int pos = t < g.tile + g.count ? (first / CTILE + t) * CTILE + (lane << c.log_page) : len;
        return lane < (CTILE >> c.log_page) && pos < len ? cache_page(c, g.b, pos >> c.log_page, 0, status) : -1;
      };
      int page = page_of(g.tile);
      for (int t = g.tile; t < g.tile + g.count; ++t, ++i) {
        const int page_next = page_of(t + 1), st = i % NST;
        const uint32_t load = bytes * (uint32_t)__popc(__ballot_sync(0xFFFFFFFFu, page >= 0));
        const size_t where = (size_t)max(page, 0) * c.kv + g.head;
        const float ks = page >= 0 ? c.ks[where] : 0.f;
        if (i >= NST) wait(&k_empty[st], i / NST - 1);
        if (!ok) break;
        if (lane == 0) mbar_expect_tx(&k_full[st], load);
        __syncwarp();
        if (page >= 0) tma_rows(k_ring + st * PL::KEYS + lane * bytes, &kmap, (int)where << c.log_page, &k_full[st]);
        if (lane < 8) key_scale[i % NSC][lane] = ks;
        __syncwarp();
        if (lane == 0) mbar_arrive(&sc_bar[i % NSC]);
        page = page_next;
      }
    }
    if (!ok) {
      if (lane == 0) atomicOr(status, STATUS_TIMEOUT);
      for (int k = max(0, i - NST); k < i; ++k) mbar_wait(&k_full[k % NST], (k / NST) & 1, wait_ns);
    }
  } else if (warp == 13) {
    // ---------------- MMA ------------------------------------------------------------------------------------------------
    const uint32_t u_tmem = __shfl_sync(0xFFFFFFFFu, tmem, 0);
    constexpr uint32_t idesc = cache_idesc(128, N, 0, 0);
    int i = 0;
    for (int seg = 0; ok && next(g); ++seg) {
      wait(&q_bar[seg & 1], seg >> 1);
      const uint64_t bd = cache_desc<DIM>(q_base + (uint32_t)(seg & 1) * PL::Q_BYTES);
      for (int t = 0; t < g.count; ++t, ++i) {
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
    }
    if (!ok) {
      if (lane == 0) atomicOr(status, STATUS_TIMEOUT);
      mma_commit(&drain_bar);
      mbar_wait(&drain_bar, 0, wait_ns);
    }
  } else if (warp >= 8) {
    // ---------------- queries ----------------------------------------------------------------------------------------------
    const int qt = tid - 256;
    constexpr int LANES = DIM / 8, AT_ONCE = 128 / LANES, PASSES = (RC + AT_ONCE - 1) / AT_ONCE;
    const int piece = qt % LANES;
    for (int seg = 0; ok && next(g); ++seg) {
      const int buf = seg & 1;
      const int2 r = cache_rows(cu, g.b, rows, status);
      const int len = cache_length(c, g.b, status);
      int h, m;
      Raw8<T> raw[PASSES];                             // all in flight at once
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        const int row = row_of(g, r, g.chunk * RC + p * AT_ONCE + qt / LANES, h, m);
        if (row >= 0) raw[p].load(q + (long long)row * q_stride + (long long)h * DIM + piece * 8);
        else raw[p].clear();
      }
      float base = 0.f;
      if (qt < RC) {
        const int row = row_of(g, r, g.chunk * RC + qt, h, m);
        if (row >= 0) base = lse[(long long)row * heads + h] * 1.4426950408889634f;
      }
      if (seg >= 2) wait(&q_free[buf], (seg >> 1) - 1);
      float scale[PASSES];
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        float f[8];
        raw[p].get(f);
        scale[p] = query_scale<DIM>(f);
      }
      // (no branch between the passes unless the last one is not full, so that their chains of conversions overlap)
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        const int x = p * AT_ONCE + qt / LANES;
        float f[8];
        raw[p].get(f);
        if (PASSES * AT_ONCE > RC && x >= RC) continue;
        store_query<DIM, NT>(f, scale[p], q_base + (uint32_t)buf * PL::Q_BYTES, x, RC, piece);
      }
      if (piece == 0) {
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
          const int x = p * AT_ONCE + qt / LANES;
          if (x < RC) row_is[buf][x >> 1][x & 1] = scale[p] * scale_log2;
        }
      }
      if (!ok) break;
      if (qt < RC) {
        const int row = row_of(g, r, g.chunk * RC + qt, h, m);
        const int3 see = seen(mask, len - (r.y - row), len);
        row_see[buf][qt] = row >= 0 ? make_int4(see.x, see.y, see.z, 0) : make_int4(0, 0, 0, 0);
        row_is[buf][qt >> 1][2 + (qt & 1)] = -base;
      }
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(&q_bar[buf]);
    }
    if (!ok && lane == 0) atomicOr(status, STATUS_TIMEOUT);
  } else {
    // ---------------- output: thread = token ---------------------------------------------------------------------------------
    const uint32_t t_lane = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const int tt = tid & 127, pg = tt >> c.log_page, turn = warp >> 2;
    int i = 0;
    for (int seg = 0; ok && next(g); ++seg) {
      const int buf = seg & 1;
      wait(&q_bar[buf], seg >> 1);
      if (!ok) break;
      const int n_x = min(RC, n_text * group - g.chunk * RC);
      // tokens that all text rows see (the first sees least ahead, the last least behind; a row that is not there sees nothing)
      const int2 r = cache_rows(cu, g.b, rows, status);
      const int len = cache_length(c, g.b, status);
      const int in_hi = r.y - r.x >= n_text ? seen(mask, len - n_text, len).z : 0, in_lo = seen(mask, len - 1, len).y;
      float* const to = weights + (((long long)g.b * heads + g.head * group) * n_text + g.chunk * RC) * count - first;
      for (int t = g.tile; t < g.tile + g.count; ++t, ++i) {
        if ((i & 1) != turn) continue;
        const int base = (first / CTILE + t) * CTILE, j = base + tt;
        wait(&sc_bar[i % NSC], i / NSC);
        const float ks = key_scale[i % NSC][pg];
        wait(&s_bar[i & 1], i >> 1);
        if (!ok) break;
        ctc_fence_after();
        const bool edge = base < in_lo || base > in_hi - CTILE, mine = j >= first && j < first + count;
#pragma unroll 1
        for (int x = 0; x < n_x; x += 16) {
          float2 s[8];                                 // sums of the terms times the page's scale, smallest term first
          {
            float f[16];
            ctmem_ld16(t_lane + (uint32_t)(i & 1) * N + (NT - 1) * RC + x, f);
#pragma unroll
            for (int u = NT - 2; u >= 0; --u) {
              float e[16];
              ctmem_ld16(t_lane + (uint32_t)(i & 1) * N + u * RC + x, e);
              ctmem_wait_ld();
              const float2 by = u == NT - 2 ? make_float2(ks * 0.0625f, ks * 0.0625f) : make_float2(0.0625f, 0.0625f);
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                const float2 low = u == NT - 2 ? make_float2(f[2 * k], f[2 * k + 1]) : s[k];
                s[k] = fma2(low, by, mul2(make_float2(e[2 * k], e[2 * k + 1]), make_float2(ks, ks)));
              }
            }
          }
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float4 is = *reinterpret_cast<const float4*>(row_is[buf][(x >> 1) + k]);
            s[k] = fma2(s[k], make_float2(is.x, is.y), make_float2(is.z, is.w));
            s[k] = make_float2(ex2(s[k].x), ex2(s[k].y));
          }
          if (edge) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const int4 e0 = row_see[buf][x + 2 * k], e1 = row_see[buf][x + 2 * k + 1];
              s[k].x = j < e0.z && (j >= e0.y || j < e0.x) ? s[k].x : 0.f;
              s[k].y = j < e1.z && (j >= e1.y || j < e1.x) ? s[k].y : 0.f;
            }
          }
          if (mine) {
            uint32_t where = (uint32_t)x * (uint32_t)count + (uint32_t)j;
            if (x + 16 <= n_x) {
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                to[where] = s[k].x; where += (uint32_t)count;
                to[where] = s[k].y; where += (uint32_t)count;
              }
            } else {
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                if (x + 2 * k < n_x) to[where] = s[k].x;
                where += (uint32_t)count;
                if (x + 2 * k + 1 < n_x) to[where] = s[k].y;
                where += (uint32_t)count;
              }
            }
          }
        }
        ctc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_relaxed(&s_free[i & 1]);
      }
      if (!ok) break;
      __syncwarp();
      if (lane == 0) mbar_arrive_relaxed(&q_free[buf]);
    }
    if (!ok && lane == 0) atomicOr(status, STATUS_TIMEOUT);
  }
  ctc_fence_before();
  __syncthreads();
  if (warp == 13) tmem_free(tmem, PL::TMEM);
}

}  // namespace ficoco
