// Attention over the 8-bit cache for few query rows per sequence (single tokens), on the 5th-generation tensor cores.
//
// Mathematics.  For a tile of 128 tokens and the RB query rows that share a key/value head, S^T = K Q^T and
// O^T = V^T P^T: the codes are operand A of both products (128 rows: tokens, then dimensions) as TMA brought them, the few
// query rows are the columns.  With s_j the score in units of log2 and e_j = log2 of the page's value scale, the
// running maximum is that of t_j = s_j + e_j, the weights are P_j = 2^(t_j - max), so that codes can be summed without their scale,
// and the denominator sums P_j / 2^e_j.  Rows and weights are split into NT e4m3 terms (cache_umma.cuh), one more block of
// columns each.  Every tile's O^T is added to fp32 registers.
//
// What bounds it: HBM, one byte per key or value element.  The tensor cores are idle most of the time and nothing is
// converted, so an SM needs 200 to 300 instructions per warp and tile of 32 KB.  All tiles of all (sequence, row block, head)
// items form one list which is cut into equal pieces, one per CTA (two CTAs per SM, so that one's softmax runs under the other's
// loads): ragged lengths balance by themselves.  An item that is cut leaves partial results; the CTA that finishes
// it last joins them in the order of the list, so the result does not depend on who that was.
//
// Roles: warps 0-3 softmax and epilogue (thread = token, then dimension), warp 4 TMA and page scales, warp 5 MMA.  Tile i's
// scores are computed while tile i - 1's weights are multiplied.
#pragma once
#include "cache_umma.cuh"

namespace ficoco {

constexpr int STEP_THREADS = 192;
constexpr int STEP_MAX_PARTS = 64;         // most pieces that an item is cut into

// One sequence of the call, in tiles.
struct StepSeq {
  int len, row0, n_rows, blocks, t_sink, t0, nt;
};
__device__ __forceinline__ StepSeq step_seq(const CacheView& c, const int* cu, int rows, int group, int rb, const MaskRule& mask,
                                            int b, unsigned* status) {
  StepSeq s;
  const int2 r = cache_rows(cu, b, rows, status);
  s.row0 = r.x;
  s.n_rows = r.y - r.x;
  s.len = s.n_rows > 0 ? cache_length(c, b, status) : 0;
  s.blocks = (int)(((long long)s.n_rows * group + rb - 1) / rb);
  // tokens that some row sees: the first sinks and everything from the first row's window on
  const int lo = mask.window > 0 ? min(max(0, s.len - s.n_rows - mask.window + 1), s.len) : 0;
  s.t0 = lo / CTILE;
  s.t_sink = min((min(mask.sinks, lo) + CTILE - 1) / CTILE, s.t0);
  s.nt = max(1, s.t_sink + (s.len + CTILE - 1) / CTILE - s.t0);
  return s;
}

// A CTA's piece of the list, one item's tiles after the other.
struct StepSeg {
  int b, head, block, tile, count;         // item and its tiles [tile, tile + count)
  StepSeq s;
};
struct StepWalk {
  long long at, end;                       // in the list
  long long first;                         // where sequence b starts in it
  int b;
  StepSeq s;
};
__device__ __forceinline__ bool step_next(StepWalk& w, StepSeg& g, const CacheView& c, const int* cu, int rows, int group, int rb,
                                          const MaskRule& mask, unsigned* status) {
  if (w.at >= w.end) return false;
  for (;;) {
    const long long size = (long long)w.s.blocks * c.kv * w.s.nt;
    if (w.at < w.first + size || w.b + 1 >= c.batch) break;
    w.first += size;
    w.s = step_seq(c, cu, rows, group, rb, mask, ++w.b, status);
  }
  const long long off = w.at - w.first;
  const int item = (int)(off / w.s.nt);
  g.b = w.b;
  g.s = w.s;
  g.head = item % c.kv;
  g.block = item / c.kv;
  g.tile = (int)(off - (long long)item * w.s.nt);
  g.count = (int)min((long long)(w.s.nt - g.tile), w.end - w.at);
  w.at += g.count;
  return true;
}
__device__ __forceinline__ int step_token0(const StepSeq& s, int tile) {      // first token of a tile of the item
  return (tile < s.t_sink ? tile : tile - s.t_sink + s.t0) * CTILE;
}

template <int DIM, int NT, int RB>
struct StepPlan {
  static constexpr int N = NT * RB;                                  // columns of both products
  static constexpr int STAGE = 2 * CTILE * DIM;                      // keys and values of a tile
  static constexpr int Q_BYTES = (N * DIM + 1023) / 1024 * 1024, P_BYTES = N * CTILE;
  static constexpr int ROOM = 112 * 1024 - 2048;                     // half an SM's shared memory, less what is static
  static constexpr int STAGES_FIT = (ROOM - 1024 - 2 * (Q_BYTES + P_BYTES)) / STAGE;
  static constexpr int STAGES = STAGES_FIT > 6 ? 6 : STAGES_FIT;
  static constexpr int SMEM = 1024 + STAGES * STAGE + 2 * (Q_BYTES + P_BYTES);
  static constexpr int TMEM = 4 * N <= 64 ? 64 : 4 * N <= 128 ? 128 : 256;
  static constexpr int PART = RB * (DIM + 2);                        // floats of a partial result
  static_assert(STAGES >= 2 && 4 * N <= 256 && N % 16 == 0, "two CTAs per SM");
};

template <class T, int DIM, int NT, int RB>
__global__ void __launch_bounds__(STEP_THREADS, 2) k_cache_step(
    const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap, const CacheView c,
    const T* __restrict__ q, const int* __restrict__ cu, T* __restrict__ out, float* __restrict__ lse, long long q_stride,
    float scale_log2, int rows, int heads, const MaskRule mask, int* __restrict__ counters, float* __restrict__ partials,
    unsigned* __restrict__ status, unsigned long long wait_ns) {
  using PL = StepPlan<DIM, NT, RB>;
  constexpr int N = PL::N, NST = PL::STAGES;
  extern __shared__ unsigned char step_raw[];
  __shared__ uint64_t full_bar[NST], empty_bar[NST], q_bar[2], s_bar[2], p_bar[2], o_bar[2], drain_bar;
  __shared__ uint32_t tmem_s;
  __shared__ float page_scale[NST][3][8];              // key scale, log2 of the value scale, 1 / value scale
  __shared__ __align__(16) float wmax[2][4][RB];
  __shared__ float lred[4][RB];
  __shared__ float q_scale[2][RB];
  __shared__ int2 row_see[2][RB];                      // tokens [x, y) of a row (and its sinks)
  __shared__ long long scan[STEP_THREADS / 32][2], start_s[4];
  __shared__ int scan_b, failed, last_s;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t ring = (smem_u32(step_raw) + 1023u) & ~1023u;
  const uint32_t q_base = ring + NST * PL::STAGE, p_base = q_base + 2 * PL::Q_BYTES;
  const int group = heads / c.kv;
  if (tid == 0) {
    for (int s = 0; s < NST; ++s) { mbar_init(&full_bar[s], 2); mbar_init(&empty_bar[s], 1); }
    for (int s = 0; s < 2; ++s) { mbar_init(&q_bar[s], 128); mbar_init(&s_bar[s], 1); mbar_init(&p_bar[s], 128); mbar_init(&o_bar[s], 1); }
    mbar_init(&drain_bar, 1);
    scan_b = -1;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 5) tmem_alloc(&tmem_s, PL::TMEM);
  grid_dep_wait();
  if (tid == 0) failed = (*reinterpret_cast<const volatile unsigned*>(status) & STATUS_TIMEOUT) ? 1 : 0;

  // ---- this CTA's piece of the list: a thread sums the tiles of a run of sequences -----------------------------------------
  const int per = (c.batch + STEP_THREADS - 1) / STEP_THREADS, b_lo = min(tid * per, c.batch), b_hi = min(b_lo + per, c.batch);
  long long mine = 0, most = 0;
  for (int b = b_lo; b < b_hi; ++b) {
    const StepSeq s = step_seq(c, cu, rows, group, RB, mask, b, status);
    mine += (long long)s.blocks * c.kv * s.nt;
    most = max(most, (long long)(s.blocks > 0 ? s.nt : 0));
  }
  long long upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long v = __shfl_up_sync(0xFFFFFFFFu, upto, o);
    if (lane >= o) upto += v;
    most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
  }
  if (lane == 31) { scan[warp][0] = upto; scan[warp][1] = most; }
  ctc_fence_before();
  __syncthreads();
  ctc_fence_after();
  grid_dep_launch();       // behind the barrier: a dependent that took this CTA's TMEM first would wait for it for ever
  const uint32_t tmem = tmem_s;
  long long total = 0, nt_most = 0;
#pragma unroll
  for (int w = 0; w < STEP_THREADS / 32; ++w) {
    if (w < warp) upto += scan[w][0];
    total += scan[w][0];
    nt_most = max(nt_most, scan[w][1]);
  }
  // CTAs that get a piece: no more than tiles, nor so many that the longest item would be cut into more than STEP_MAX_PARTS
  long long n_cta = min((long long)gridDim.x, total);
  if (nt_most > 0) n_cta = max(1ll, min(n_cta, (STEP_MAX_PARTS - 1) * total / nt_most));
  StepWalk walk;
  walk.at = blockIdx.x < n_cta ? total * blockIdx.x / n_cta : 0;
  walk.end = blockIdx.x < n_cta ? total * (blockIdx.x + 1) / n_cta : 0;
  if (walk.at < walk.end && walk.at >= upto - mine && walk.at < upto) {      // one thread's run holds the start
    long long at = upto - mine;
    int b = b_lo;
    for (; b + 1 < b_hi; ++b) {
      const StepSeq s = step_seq(c, cu, rows, group, RB, mask, b, status);
      const long long size = (long long)s.blocks * c.kv * s.nt;
      if (walk.at < at + size) break;
      at += size;
    }
    start_s[0] = at;
    scan_b = b;
  }
  __syncthreads();
  const bool idle = walk.at >= walk.end || failed != 0 || scan_b < 0;
  if (!idle) {
    walk.b = scan_b;
    walk.first = start_s[0];
    walk.s = step_seq(c, cu, rows, group, RB, mask, walk.b, status);
  } else {
    walk.at = walk.end = 0;
  }
  bool ok = true;

  if (warp == 4) {
    // ---------------- TMA: lane p brings page p of a tile ----------------------------------------------------------------
    StepSeg g;
    int i = 0, st = 0;
    uint32_t par = 1;
    while (ok && step_next(walk, g, c, cu, rows, group, RB, mask, status)) {
      for (int t = g.tile; t < g.tile + g.count; ++t, ++i) {
        const int base = step_token0(g.s, t), left = min(CTILE, g.s.len - base);
        const int pages = left > 0 ? (left + c.page - 1) >> c.log_page : 0;
        int page = 0;
        if (lane < pages) page = cache_page(c, g.b, (base >> c.log_page) + lane, 0, status);
        if (i >= NST) ok = __all_sync(0xFFFFFFFFu, mbar_wait(&empty_bar[st], par, wait_ns));
        if (!ok) break;
        const uint32_t bytes = (uint32_t)(c.page * DIM);
        if (lane == 0) mbar_expect_tx(&full_bar[st], 2u * bytes * (uint32_t)pages);
        __syncwarp();
        const size_t at = (size_t)page * c.kv + g.head;
        if (lane < pages) {
          const uint32_t dst = ring + (uint32_t)st * PL::STAGE + (uint32_t)lane * bytes;
          tma_rows(dst, &kmap, (int)(at << c.log_page), &full_bar[st]);
          tma_rows(dst + CTILE * DIM, &vmap, (int)(at << c.log_page), &full_bar[st]);
          const float sv = c.vs[at];
          page_scale[st][0][lane] = c.ks[at];
          page_scale[st][1][lane] = log2f(sv);
          page_scale[st][2][lane] = 1.0f / sv;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&full_bar[st]);
        if (++st == NST) { st = 0; par ^= 1u; }
      }
    }
    if (!ok) {
      atomicOr(status, STATUS_TIMEOUT);
      // no copy outlives the CTA: the tiles asked for last
      for (int k = max(0, i - NST); k < i; ++k) mbar_wait(&full_bar[k % NST], (k / NST) & 1, wait_ns);
      failed = 1;
    }
  } else if (warp == 5) {
    // ---------------- MMA: scores of tile i + 1 go out before the weights of tile i are waited for ------------------------
    const uint32_t u_tmem = __shfl_sync(0xFFFFFFFFu, tmem, 0);
    constexpr uint32_t id_s = cache_idesc(128, N, 0, 0), id_o = cache_idesc(DIM, N, 1, 0);
    StepSeg g;
    int seg = -1, left = 0, st = 0, st_prev = 0;
    uint32_t par = 0;
    for (int i = 0;; ++i) {
      bool more = true;
      if (left == 0) {
        more = step_next(walk, g, c, cu, rows, group, RB, mask, status);
        if (more) {
          ++seg;
          left = g.count;
          ok = __all_sync(0xFFFFFFFFu, mbar_wait(&q_bar[seg & 1], (seg >> 1) & 1, wait_ns));
          if (!ok) break;
        }
      }
      if (more) {
        --left;
        ok = __all_sync(0xFFFFFFFFu, mbar_wait(&full_bar[st], par, wait_ns));
        if (!ok) break;
        ctc_fence_after();
        const uint32_t a = ring + (uint32_t)st * PL::STAGE, b = q_base + (uint32_t)(seg & 1) * PL::Q_BYTES;
        const uint64_t ad = cache_desc<DIM>(a), bd = cache_desc<DIM>(b);
#pragma unroll
        for (int k = 0; k < DIM / 32; ++k) mma_f8(u_tmem + (uint32_t)(i & 1) * N, ad + 2 * k, bd + 2 * k, id_s, k > 0);
        mma_commit(&s_bar[i & 1]);
      }
      if (i > 0) {
        const int j = i - 1;
        ok = __all_sync(0xFFFFFFFFu, mbar_wait(&p_bar[j & 1], (j >> 1) & 1, wait_ns));
        if (!ok) break;
        ctc_fence_after();
        const uint64_t ad = cache_desc<DIM>(ring + (uint32_t)st_prev * PL::STAGE + CTILE * DIM);
        const uint64_t bd = cache_desc<128>(p_base + (uint32_t)(j & 1) * PL::P_BYTES);
#pragma unroll
        for (int k = 0; k < CTILE / 32; ++k)
          mma_f8(u_tmem + 2 * N + (uint32_t)(j & 1) * N, ad + (uint64_t)(k * (32 * DIM >> 4)), bd + 2 * k, id_o, k > 0);
        mma_commit(&o_bar[j & 1]);
        mma_commit(&empty_bar[st_prev]);
      }
      if (!more) break;
      st_prev = st;
      if (++st == NST) { st = 0; par ^= 1u; }
    }
    if (!ok) {
      atomicOr(status, STATUS_TIMEOUT);
      mma_commit(&drain_bar);
      mbar_wait(&drain_bar, 0, wait_ns);
      failed = 1;
    }
  } else {
    // ---------------- softmax: thread = token of the tile, then dimension of the output ------------------------------------
    const uint32_t t_lane = tmem + ((uint32_t)(warp * 32) << 16);
    constexpr int LANES = DIM / 8, PASS_ROWS = 128 / LANES, PASSES = (RB + PASS_ROWS - 1) / PASS_ROWS;
    const int q_chunk = tid % LANES, q_row = tid / LANES;
    float qf[PASSES][8];
    // rows of an item: row x of block k is head x % group of the sequence's row x / group
    auto load_q = [&](const StepSeg& g) {
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        const long long x = (long long)g.block * RB + p * PASS_ROWS + q_row;
        const int i = (int)(x / group), h = g.head * group + (int)(x - (long long)i * group);
        const bool on = p * PASS_ROWS + q_row < RB && i < g.s.n_rows;
        if (on) load8(q + (long long)(g.s.row0 + i) * q_stride + (long long)h * DIM + q_chunk * 8, qf[p]);
        else {
#pragma unroll
          for (int j = 0; j < 8; ++j) qf[p][j] = 0.f;
        }
      }
    };
    auto put_q = [&](const StepSeg& g, int buf) {
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        const int r = p * PASS_ROWS + q_row;
        if (PASSES * PASS_ROWS > RB && r >= RB) continue;      // (whole warps: RB is a multiple of a warp's rows)
        const float s = store_query<DIM, NT>(qf[p], q_base + (uint32_t)buf * PL::Q_BYTES, r, RB, q_chunk);
        if (q_chunk == 0) q_scale[buf][r] = s * scale_log2;
      }
      if (tid < RB) {
        const long long x = (long long)g.block * RB + tid;
        const int i = (int)min(x / group, (long long)g.s.n_rows);
        const int3 see = seen(mask, g.s.len - g.s.n_rows + i, g.s.len);
        row_see[buf][tid] = i < g.s.n_rows ? make_int2(see.y, see.z) : make_int2(0, 0);
      }
      fence_proxy_async();
      mbar_arrive(&q_bar[buf]);
    };
    StepSeg g, g_next;
    bool have = step_next(walk, g, c, cu, rows, group, RB, mask, status);
    long long seg_at = walk.at;                                // end of segment g in the list
    if (have) { load_q(g); put_q(g, 0); }
    cta_sync(1, 128);                                          // the rows' scales and masks are in shared memory
    int i = 0, st = 0, seg = 0;
    uint32_t par = 0;
    float m[RB], l[RB], acc[RB];
    while (have) {
      seg_at = walk.at;
      const bool have_next = step_next(walk, g_next, c, cu, rows, group, RB, mask, status);
      if (have_next) load_q(g_next);
      const int buf_q = seg & 1;
#pragma unroll
      for (int r = 0; r < RB; ++r) { m[r] = -CUDART_INF_F; l[r] = 0.f; acc[r] = 0.f; }
      // a tile inside [in_lo, in_hi) is seen by every row of the item
      const int i_first = (int)((long long)g.block * RB / group);
      const int i_last = (int)min(((long long)g.block * RB + RB - 1) / group, (long long)g.s.n_rows - 1);
      const int in_hi = seen(mask, g.s.len - g.s.n_rows + i_first, g.s.len).z;
      const int in_lo = seen(mask, g.s.len - g.s.n_rows + i_last, g.s.len).y;
      for (int t = g.tile; t < g.tile + g.count; ++t, ++i) {
        const int base = step_token0(g.s, t), buf = i & 1;
        if (ok) ok = mbar_wait(&full_bar[st], par, wait_ns);   // (page scales; and values, where they are cleared below)
        const int pg = tid >> c.log_page;
        const bool token = base + tid < g.s.len;               // (pages behind the last one have no scales)
        const float ks = page_scale[st][0][pg], ve = page_scale[st][1][pg], vi = token ? page_scale[st][2][pg] : 0.f;
        if (ok) ok = mbar_wait(&s_bar[buf], (i >> 1) & 1, wait_ns);
        ctc_fence_after();
        float s[N];
#pragma unroll
        for (int n = 0; n < N; n += 16) ctmem_ld16(t_lane + (uint32_t)buf * N + n, s + n);
        ctmem_wait_ld();
        const bool edge = base < in_lo || base + CTILE > in_hi;
        const int j = base + tid;
#pragma unroll
        for (int r = 0; r < RB; ++r) {
          float x = s[(NT - 1) * RB + r];
#pragma unroll
          for (int u = NT - 2; u >= 0; --u) x = fmaf(x, 0.0625f, s[u * RB + r]);
          s[r] = fmaf(x, q_scale[buf_q][r] * ks, ve);
        }
        if (edge) {
#pragma unroll
          for (int r = 0; r < RB; ++r) {
            const int2 see = row_see[buf_q][r];
            const bool on = j < see.y && (j >= see.x || j < mask.sinks);
            s[r] = on ? s[r] : -CUDART_INF_F;
          }
          if (!token) {                                        // no token: whatever the slot holds must not meet a weight of 0
            const uint32_t v = ring + (uint32_t)st * PL::STAGE + CTILE * DIM + tid * DIM;
#pragma unroll
            for (int x = 0; x < DIM; x += 16) st_shared16(v + x, 0u, 0u, 0u, 0u);
          }
        }
#pragma unroll
        for (int r = 0; r < RB; ++r) {
          const float x = warp_max(s[r]);
          if (lane == r) wmax[buf][warp][r] = x;
        }
        // a wait that ran out anywhere ends the loop for all 128 threads
        if (cta_sync_or(1, 128, !ok)) { ok = false; break; }
        float corr[RB];
#pragma unroll
        for (int r = 0; r < RB; ++r) {
          const float x = fmaxf(fmaxf(wmax[buf][0][r], wmax[buf][1][r]), fmaxf(wmax[buf][2][r], wmax[buf][3][r]));
          const float mn = fmaxf(m[r], x), ref = mn == -CUDART_INF_F ? 0.f : mn;
          corr[r] = ex2(m[r] - ref);
          m[r] = mn;
          s[r] = ex2(s[r] - ref);
          l[r] = fmaf(l[r], corr[r], s[r] * vi);
        }
        const uint32_t p = p_base + (uint32_t)buf * PL::P_BYTES;
#pragma unroll
        for (int r = 0; r < RB; r += 2) {
          uint32_t code[NT];
          split_pair<NT>(s[r] * 256.f, s[r + 1] * 256.f, code);
#pragma unroll
          for (int u = 0; u < NT; ++u) {
            const int n = u * RB + r;
            st_shared1(p + n * 128 + ((((tid >> 4) ^ n) & 7) << 4) + (tid & 15), code[u] & 0xFFu);
            st_shared1(p + (n + 1) * 128 + ((((tid >> 4) ^ (n + 1)) & 7) << 4) + (tid & 15), code[u] >> 8);
          }
        }
        fence_proxy_async();
        ctc_fence_before();
        mbar_arrive(&p_bar[buf]);
        if (t == g.tile) {
          if (have_next) put_q(g_next, buf_q ^ 1);
        } else {                                               // what the tile before this one added
          if (ok) ok = mbar_wait(&o_bar[buf ^ 1], ((i - 1) >> 1) & 1, wait_ns);
          ctc_fence_after();
          float o[N];
#pragma unroll
          for (int n = 0; n < N; n += 16) ctmem_ld16(t_lane + 2 * N + (uint32_t)(buf ^ 1) * N + n, o + n);
          ctmem_wait_ld();
#pragma unroll
          for (int r = 0; r < RB; ++r) {
            float x = o[(NT - 1) * RB + r];
#pragma unroll
            for (int u = NT - 2; u >= 0; --u) x = fmaf(x, 0.0625f, o[u * RB + r]);
            acc[r] = (acc[r] + x) * corr[r];
          }
          ctc_fence_before();
        }
        if (++st == NST) { st = 0; par ^= 1u; }
      }
      if (!ok) break;
      if (ok) ok = mbar_wait(&o_bar[(i - 1) & 1], ((i - 1) >> 1) & 1, wait_ns);
      ctc_fence_after();
      {
        float o[N];
#pragma unroll
        for (int n = 0; n < N; n += 16) ctmem_ld16(t_lane + 2 * N + (uint32_t)((i - 1) & 1) * N + n, o + n);
        ctmem_wait_ld();
#pragma unroll
        for (int r = 0; r < RB; ++r) {
          float x = o[(NT - 1) * RB + r];
#pragma unroll
          for (int u = NT - 2; u >= 0; --u) x = fmaf(x, 0.0625f, o[u * RB + r]);
          acc[r] += x;
        }
        ctc_fence_before();
      }
#pragma unroll
      for (int r = 0; r < RB; ++r) {
        const float x = warp_sum(l[r]);
        if (lane == 0) lred[warp][r] = x;
      }
      if (cta_sync_or(1, 128, !ok)) { ok = false; break; }
#pragma unroll
      for (int r = 0; r < RB; ++r) l[r] = (lred[0][r] + lred[1][r]) + (lred[2][r] + lred[3][r]);
      // (M = 64 accumulators lie in the first sixteen lanes of each warp)
      const bool has_dim = DIM == 128 || lane < 16;
      const int d = DIM == 128 ? tid : warp * 16 + lane;
      const int x0 = g.block * RB, nr = (int)min((long long)RB, (long long)g.s.n_rows * group - x0);
      if (g.count == g.s.nt) {
#pragma unroll
        for (int r = 0; r < RB; ++r) {
          if (r < nr) {
            const int ri = (x0 + r) / group, h = g.head * group + (x0 + r) - ri * group;
            const long long at = (long long)(g.s.row0 + ri) * heads + h;
            if (has_dim) store1(out + at * DIM + d, l[r] > 0.f || l[r] != l[r] ? acc[r] * (0.00390625f / l[r]) : 0.f);
            if (lse != nullptr && tid == r) lse[at] = l[r] > 0.f || l[r] != l[r] ? (m[r] + log2f(l[r])) * 0.69314718055994531f : -CUDART_INF_F;
          }
        }
      } else {
        // A cut item.  Its first piece is the last one of CTA `owner`, the others are the first ones of the CTAs behind it.
        const long long item0 = seg_at - g.count - g.tile, item1 = item0 + g.s.nt;
        auto cta_of = [&](long long x) { return (int)(((x + 1) * n_cta + total - 1) / total - 1); };
        const int owner = cta_of(item0), parts = cta_of(item1 - 1) - owner + 1;
        float* mine_p = partials + ((size_t)blockIdx.x * 2 + (g.tile == 0 ? 1 : 0)) * PL::PART;
#pragma unroll
        for (int r = 0; r < RB; ++r) {
          if (has_dim) __stcg(mine_p + r * DIM + d, acc[r]);
          if (tid == r) { __stcg(mine_p + RB * DIM + r, m[r]); __stcg(mine_p + RB * DIM + RB + r, l[r]); }
        }
        cta_sync(1, 128);
        if (tid == 0) last_s = atom_acq_rel_add(&counters[owner], 1) == parts - 1;
        cta_sync(1, 128);
        if (last_s) {
          if (tid == 0) counters[owner] = 0;
          __threadfence();
          auto part = [&](int k) { return partials + ((size_t)(owner + k) * 2 + (k == 0 ? 1 : 0)) * PL::PART; };
          for (int u = tid; u < nr * (DIM / 4); u += 128) {
            const int r = u / (DIM / 4), d4 = (u % (DIM / 4)) * 4;
            float top = -CUDART_INF_F;
#pragma unroll 8
            for (int k = 0; k < parts; ++k) top = fmaxf(top, __ldcg(part(k) + RB * DIM + r));
            const float ref = top == -CUDART_INF_F ? 0.f : top;
            float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
            float ls = 0.f;
#pragma unroll 8
            for (int k = 0; k < parts; ++k) {
              const float* pk = part(k);
              const float w = ex2(__ldcg(pk + RB * DIM + r) - ref);
              const float4 v = __ldcg(reinterpret_cast<const float4*>(pk + r * DIM + d4));
              ls = fmaf(w, __ldcg(pk + RB * DIM + RB + r), ls);
              a.x = fmaf(w, v.x, a.x); a.y = fmaf(w, v.y, a.y); a.z = fmaf(w, v.z, a.z); a.w = fmaf(w, v.w, a.w);
            }
            const bool some = ls > 0.f || ls != ls;
            const float inv = some ? 0.00390625f / ls : 0.f;
            const int ri = (x0 + r) / group, h = g.head * group + (x0 + r) - ri * group;
            const long long at = (long long)(g.s.row0 + ri) * heads + h;
            T* o = out + at * DIM + d4;
            store1(o, some ? a.x * inv : 0.f); store1(o + 1, some ? a.y * inv : 0.f);
            store1(o + 2, some ? a.z * inv : 0.f); store1(o + 3, some ? a.w * inv : 0.f);
            if (lse != nullptr && d4 == 0) lse[at] = some ? (top + log2f(ls)) * 0.69314718055994531f : -CUDART_INF_F;
          }
        }
      }
      g = g_next;
      have = have_next;
      ++seg;
    }
    if (!ok) {
      if (tid == 0) { atomicOr(status, STATUS_TIMEOUT); failed = 1; }
    }
  }
  ctc_fence_before();
  __syncthreads();
  if (warp == 5) tmem_free(tmem, PL::TMEM);
}

}  // namespace ficoco
