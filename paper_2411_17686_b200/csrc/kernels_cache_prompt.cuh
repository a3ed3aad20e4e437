// Attention over the 8-bit cache for many bf16 query rows per sequence (prompts and chunks of them), on the 5th-generation tensor
// cores.
//
// Mathematics.  Rows of a sequence that share a key/value head are packed, 128 to a tile (row x = query x / group, head x % group of the
// group), so that a tile reads its keys and values once for all heads of the group.  S = Q K^T per tile of 128 tokens: the keys' codes
// as they lie in memory against two e4m3 terms of the query rows at one scale (cache_umma.cuh).  t = log2 score + log2 of the
// page's value scale; P = 2^(t - ref) in fp16 (2^-11, where two e4m3 terms would hold 2^-8 and cost twice the conversions), the
// values' codes converted to fp16, which is exact; the denominator sums P / value scale in fp32.  ref lies 2^7 below the largest t
// of a tile of tokens and is left there while a tile's largest P stays in [2^-5, 2^15] (fp16 ends at 2^16 and 2^-24), so that O is rarely
// rescaled: fp16 holds a weight to 2^-11, and to 2^-20 of the largest one of its tile.  It follows the tiles down as well as up: behind a
// dominant first token, whose value is near zero, a reference that stays at the running maximum loses the bits of all others (from 2^-14 of it
// on, all of them at 2^-25).  Not further than 2^16 below the highest it was, so that sums and denominators cannot overflow.
//
// What bounds it: the tensor cores and the exponentials, which take about the same time: two row tiles per CTA take turns, one's
// softmax runs under the other's products.  P lies in tensor memory in the place of the scores it came from, which spares shared
// memory a third of its traffic (a product whose operands are both in shared memory runs at its 128 bytes per cycle).
//
// Roles: warps 0-7 and 8-15 softmax and epilogue of the two tiles (thread = row and half of the tokens, scores in registers; a warp and
// its partner exchange maxima), warps 16 and 17 convert values, warp 18 TMA and page scales, warp 19 MMA.  One CTA per SM and work item; a
// sequence's last rows, which see most, go first.
//
// Measured: four causal prompts of 2500 to 2944 rows over up to 4000 tokens, 32 heads of 128: 472 us, 0.67 PFLOP/s of what is seen.  A tile
// of tokens takes 4800 cycles for both row tiles, its products 2048: the chain scores, weights, products of one row tile (3500
// cycles of softmax with both tiles' warps on the schedulers) is what is left; with a quarter of the exponentials it would be 376 us.
// A reference that only rises is 464 us.
#pragma once
#include "cache_umma.cuh"

namespace ficoco {

constexpr int PROMPT_THREADS = 640;
constexpr int PROMPT_ROWS = 256;             // rows per CTA, two tiles

// tcgen05.mma kind::f16 with A (fp16) in tensor memory.
__device__ __forceinline__ void mma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "elect.sync _|q, 0xFFFFFFFF;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void ctmem_ld32(uint32_t taddr, float (&f)[32]) {
  uint32_t* r = reinterpret_cast<uint32_t*>(f);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, "
      "%27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
        "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
        "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr) : "memory");
}
__device__ __forceinline__ void ctmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void ctmem_st32(uint32_t taddr, const float* f) {
  const uint32_t* r = reinterpret_cast<const uint32_t*>(f);
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, "
      "%28, %29, %30, %31, %32};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
        "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
        "r"(r[30]), "r"(r[31]) : "memory");
}
__device__ __forceinline__ void ctmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t to_f16x2(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
__device__ __forceinline__ uint32_t f16x2_of(uint32_t codes) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)codes));
  return h;
}

// The bits [lo, hi) of a word, for any lo and hi.
__device__ __forceinline__ uint32_t bits(int lo, int hi) {
  const uint32_t below_hi = hi >= 32 ? ~0u : hi <= 0 ? 0u : (1u << hi) - 1u;
  return lo <= 0 ? below_hi : lo >= 32 ? 0u : below_hi & ~((1u << lo) - 1u);
}

template <int DIM>
struct PromptPlan {
  static constexpr int Q_TERM = 128 * DIM, Q_TILE = 2 * Q_TERM;      // two e4m3 terms of a row tile
  static constexpr int CODES = CTILE * DIM;                          // keys or values of a tile of tokens
  static constexpr int V16 = 2 * CODES;
  static constexpr int K_ST = 3, V_ST = 2, V16_ST = 2, SC_ST = 4;
  static constexpr int SMEM = 1024 + 2 * Q_TILE + K_ST * CODES + V_ST * CODES + V16_ST * V16;
  static_assert(PROMPT_ROWS * DIM * 2 <= V16_ST * V16, "the query rows' place");
  static_assert(SMEM + 4096 <= 227 * 1024, "one CTA per SM");
};

template <int DIM>
__global__ void __launch_bounds__(PROMPT_THREADS, 1) k_cache_prompt(
    const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap, const CacheView c,
    const __nv_bfloat16* __restrict__ q, const int* __restrict__ cu, __nv_bfloat16* __restrict__ out, float* __restrict__ lse,
    long long q_stride, float scale_log2, int rows, int heads, const MaskRule mask, unsigned* __restrict__ status,
    unsigned long long wait_ns, int extra_arrivals) {
  using PL = PromptPlan<DIM>;
  constexpr int K_ST = PL::K_ST, V_ST = PL::V_ST, V16_ST = PL::V16_ST, SC_ST = PL::SC_ST;
  extern __shared__ unsigned char prompt_raw[];
  __shared__ uint64_t k_full[K_ST], k_empty[K_ST], v_full[V_ST], v_empty[V_ST], w_full[V16_ST], w_empty[V16_ST];
  __shared__ uint64_t sc_full[SC_ST], sc_empty[SC_ST], raw_bar, q_bar, s_bar[2], p_bar[2], o_bar[2], drain_bar;
  __shared__ uint32_t tmem_s;
  __shared__ int dead_s;
  __shared__ float page_scale[SC_ST][3][8];            // key scale, log2 of the value scale, 1 / value scale
  __shared__ float q_scale[PROMPT_ROWS];
  __shared__ float half_s[2][PROMPT_ROWS];             // per half of the tokens: a tile's maxima, in the end the denominators

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t q_base = (smem_u32(prompt_raw) + 1023u) & ~1023u;
  const uint32_t k_ring = q_base + 2 * PL::Q_TILE, v_ring = k_ring + K_ST * PL::CODES, w_ring = v_ring + V_ST * PL::CODES;
  const uint32_t group = (uint32_t)(heads / c.kv);
  if (tid == 0) {
    for (int s = 0; s < K_ST; ++s) { mbar_init(&k_full[s], 1); mbar_init(&k_empty[s], 1); }
    for (int s = 0; s < V_ST; ++s) { mbar_init(&v_full[s], 1); mbar_init(&v_empty[s], 2); }
    for (int s = 0; s < V16_ST; ++s) { mbar_init(&w_full[s], 2); mbar_init(&w_empty[s], 1); }
    for (int s = 0; s < SC_ST; ++s) { mbar_init(&sc_full[s], 1); mbar_init(&sc_empty[s], 16); }
    for (int s = 0; s < 2; ++s) { mbar_init(&s_bar[s], 1); mbar_init(&p_bar[s], 8 + extra_arrivals); mbar_init(&o_bar[s], 1); }
    mbar_init(&raw_bar, PROMPT_ROWS);
    mbar_init(&q_bar, 16);
    mbar_init(&drain_bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 19) tmem_alloc(&tmem_s, 512);
  grid_dep_wait();
  if (tid == 0) dead_s = (*reinterpret_cast<const volatile unsigned*>(status) & STATUS_TIMEOUT) ? 1 : 0;

  // ---- which rows: CTA u of sequence b has rows of pair (last - u) of one head ------------------------------------------
  const int head = blockIdx.x % c.kv;
  const long long u = blockIdx.x / c.kv;
  auto unit0 = [&](int s) { return (long long)max(cu[s], 0) * group / PROMPT_ROWS + s; };
  const int b = owner_of(c.batch, unit0, u);
  const int2 r = cache_rows(cu, b, rows, status);
  const int n_rows = r.y - r.x, len = cache_length(c, b, status);
  const uint32_t packed = (uint32_t)n_rows * group;                    // rows of the sequence under this head
  const int pair = (int)((packed + PROMPT_ROWS - 1) / PROMPT_ROWS) - 1 - (int)(u - unit0(b));
  ctc_fence_before();
  __syncthreads();
  ctc_fence_after();
  grid_dep_launch();       // behind the barrier: a dependent that took this SM's TMEM first would wait for it for ever
  const uint32_t tmem = tmem_s;
  const bool work = pair >= 0 && u >= unit0(b) && !dead_s && tmem == 0;
  // ---- tiles of tokens that the rows see ----------------------------------------------------------------------------
  const uint32_t x0 = (uint32_t)max(pair, 0) * PROMPT_ROWS;
  auto query = [&](uint32_t x) { return (int)(min(x, packed - 1) / group); };      // of packed row x
  int t_sink = 0, t0 = 0, nt[2] = {0, 0};
  if (work) {
    const int first_lo = seen(mask, len - n_rows + query(x0), len).y;
    t0 = first_lo / CTILE;
    t_sink = min((min(mask.sinks, first_lo) + CTILE - 1) / CTILE, t0);
#pragma unroll
    for (int t = 0; t < 2; ++t)
      if (x0 + 128 * t < packed) {
        const int hi = seen(mask, len - n_rows + query(x0 + 128 * t + 127), len).z;
        nt[t] = max(0, t_sink + (hi + CTILE - 1) / CTILE - t0);
      }
  }
  const int n_tiles = max(nt[0], nt[1]);
  auto token0 = [&](int k) { return (k < t_sink ? k : k - t_sink + t0) * CTILE; };
  bool ok = true;                                      // the same in all lanes of a warp
  auto wait = [&](uint64_t* bar, int phase) { ok = ok && warp_wait(bar, (uint32_t)phase & 1u, wait_ns); };

  if (warp == 18) {
    // ---------------- TMA and page scales: lane p brings page p of a tile -----------------------------------------------
    const uint32_t bytes = (uint32_t)(c.page * DIM);
    auto page_of = [&](int k) {                        // this lane's page of tile k, -1: none
      const int at = k < n_tiles ? token0(k) + (lane << c.log_page) : len;
      return lane < (CTILE >> c.log_page) && at < len ? cache_page(c, b, at >> c.log_page, 0, status) : -1;
    };
    int page = page_of(0), i = 0;
    for (; i < n_tiles; ++i) {
      const int page_next = page_of(i + 1);            // a tile ahead
      const uint32_t load = bytes * (uint32_t)__popc(__ballot_sync(0xFFFFFFFFu, page >= 0));
      const size_t at = (size_t)max(page, 0) * c.kv + head;
      const float ks = page >= 0 ? c.ks[at] : 1.f, vs = page >= 0 ? c.vs[at] : 1.f;
      const int row = (int)(at << c.log_page), ks_ = i % K_ST, vs_ = i % V_ST, cs_ = i % SC_ST;
      if (i >= K_ST) wait(&k_empty[ks_], i / K_ST - 1);
      if (!ok) break;
      if (lane == 0) mbar_expect_tx(&k_full[ks_], load);
      __syncwarp();
      if (page >= 0) tma_rows(k_ring + ks_ * PL::CODES + lane * bytes, &kmap, row, &k_full[ks_]);
      if (i >= SC_ST) wait(&sc_empty[cs_], i / SC_ST - 1);
      if (ok && lane < 8) {
        page_scale[cs_][0][lane] = ks;
        page_scale[cs_][1][lane] = log2f(vs);
        page_scale[cs_][2][lane] = 1.0f / vs;
      }
      __syncwarp();
      if (ok && lane == 0) mbar_arrive(&sc_full[cs_]);
      if (i >= V_ST) wait(&v_empty[vs_], i / V_ST - 1);
      if (!ok) { mbar_wait(&k_full[ks_], (uint32_t)(i / K_ST) & 1u, wait_ns); break; }
      if (lane == 0) mbar_expect_tx(&v_full[vs_], load);
      __syncwarp();
      if (page >= 0) tma_rows(v_ring + vs_ * PL::CODES + lane * bytes, &vmap, row, &v_full[vs_]);
      page = page_next;
    }
    if (!ok) {
      if (lane == 0) atomicOr(status, STATUS_TIMEOUT);
      // no copy outlives the CTA: the tiles asked for last
      for (int k = max(0, i - K_ST); k < i; ++k) mbar_wait(&k_full[k % K_ST], (k / K_ST) & 1, wait_ns);
      for (int k = max(0, i - V_ST); k < i; ++k) mbar_wait(&v_full[k % V_ST], (k / V_ST) & 1, wait_ns);
    }
  } else if (warp == 19) {
    // ---------------- MMA: per tile of tokens, each row tile's weights times values, then its next scores ------------------
    // (all 512 columns are this CTA's, so its addresses start at 0: as a constant they stay in uniform registers)
    constexpr uint32_t u_tmem = 0;
    constexpr uint32_t id_s = cache_idesc(128, CTILE, 0, 0), id_o = cache_idesc(128, DIM, 0, 1);
    auto scores = [&](int t, int i) {
      const uint32_t qa = q_base + t * PL::Q_TILE;
      const uint64_t kd = cache_desc<DIM>(k_ring + (i % K_ST) * PL::CODES);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint64_t qd = cache_desc<DIM>(qa + e * PL::Q_TERM);
#pragma unroll
        for (int k = 0; k < DIM / 32; ++k) mma_f8(u_tmem + t * 128, qd + 2 * k, kd + 2 * k, id_s, e + k > 0);
      }
      mma_commit(&s_bar[t]);
    };
    auto sums = [&](int t, int i) {
      // fp16 values, MN-major: 64 dimensions of 128 tokens are 16 KB, eight tokens 1 KB
      const uint32_t w = w_ring + (i % V16_ST) * PL::V16;
      uint64_t wd = 0;
      wd |= (uint64_t)((w & 0x3FFFFu) >> 4);
      wd |= (uint64_t)((CTILE * 128) >> 4) << 16;
      wd |= (uint64_t)(1024 >> 4) << 32;
      wd |= (uint64_t)1 << 46;
      wd |= (uint64_t)2 << 61;
#pragma unroll
      for (int k = 0; k < CTILE / 16; ++k)
        mma_f16_ts(u_tmem + 256 + t * 128, u_tmem + t * 128 + k * 8, wd + (uint64_t)(k * (2048 >> 4)), id_o, i > 0 || k > 0);
    };
    if (n_tiles > 0) wait(&q_bar, 0);
    if (n_tiles > 0) wait(&k_full[0], 0);
    if (ok && n_tiles > 0) {
      ctc_fence_after();
      if (nt[0] > 0) scores(0, 0);
      if (nt[1] > 0) scores(1, 0);
      mma_commit(&k_empty[0]);
    }
    for (int i = 0; ok && i < n_tiles; ++i) {
      wait(&w_full[i % V16_ST], i / V16_ST);
      if (ok && i + 1 < n_tiles) wait(&k_full[(i + 1) % K_ST], (i + 1) / K_ST);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (i < nt[t]) {
          wait(&p_bar[t], i);
          if (!ok) break;
          ctc_fence_after();
          sums(t, i);
          if (i + 1 == nt[t]) mma_commit(&o_bar[t]);
        }
        if (i + 1 < nt[t]) scores(t, i + 1);
      }
      if (!ok) break;
      mma_commit(&w_empty[i % V16_ST]);
      if (i + 1 < n_tiles) mma_commit(&k_empty[(i + 1) % K_ST]);
    }
    if (!ok) {
      if (lane == 0) atomicOr(status, STATUS_TIMEOUT);
      mma_commit(&drain_bar);
      mbar_wait(&drain_bar, 0, wait_ns);
    }
  } else if (warp >= 16) {
    // ---------------- values: e4m3 -> fp16, thread = 16 dimensions of every (64 * 16 / DIM)-th token ---------------------
    constexpr int CHUNKS = DIM / 16;
    const int ct = tid - 512, ch = ct % CHUNKS;
    if (n_tiles > 0) wait(&q_bar, 0);                  // (the query rows lie where the values go)
    for (int i = 0; ok && i < n_tiles; ++i) {
      wait(&v_full[i % V_ST], i / V_ST);
      if (i >= V16_ST) wait(&w_empty[i % V16_ST], i / V16_ST - 1);
      if (!ok) break;
      const uint32_t v = v_ring + (i % V_ST) * PL::CODES, w = w_ring + (i % V16_ST) * PL::V16 + (ch >> 2) * (CTILE * 128);
      const int left = len - token0(i);                // tokens behind it: whatever the slot holds must not meet a weight of 0
      constexpr int STEP = 64 / CHUNKS;
#pragma unroll 1
      for (int j0 = ct / CHUNKS; j0 < CTILE; j0 += 4 * STEP) {
        uint32_t a[4][4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {                  // (four loads in flight: one at a time, a tile took 2800 cycles)
          const int j = j0 + e * STEP, sw = DIM == 128 ? ch ^ (j & 7) : ch ^ ((j >> 1) & 3);
          asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(a[e][0]), "=r"(a[e][1]), "=r"(a[e][2]), "=r"(a[e][3])
                       : "r"(v + j * DIM + sw * 16) : "memory");
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int j = j0 + e * STEP;
          const bool on = j < left;
#pragma unroll
          for (int x = 0; x < 4; ++x) a[e][x] = on ? a[e][x] : 0u;
          const uint32_t to = w + j * 128;
          const int c2 = (ch & 3) * 2;                 // two 16-byte pieces of the token's 128-byte row
          st_shared16(to + ((c2 ^ (j & 7)) << 4), f16x2_of(a[e][0]), f16x2_of(a[e][0] >> 16), f16x2_of(a[e][1]), f16x2_of(a[e][1] >> 16));
          st_shared16(to + (((c2 + 1) ^ (j & 7)) << 4), f16x2_of(a[e][2]), f16x2_of(a[e][2] >> 16), f16x2_of(a[e][3]), f16x2_of(a[e][3] >> 16));
        }
      }
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) { mbar_arrive(&v_empty[i % V_ST]); mbar_arrive(&w_full[i % V16_ST]); }
    }
    if (!ok && lane == 0) atomicOr(status, STATUS_TIMEOUT);
  } else {
    // ---------------- softmax: thread = row and half of the tokens ---------------------------------------------------------
    const int t = warp >> 3, half = warp >> 2 & 1, wr = warp & 3, row = t * 128 + wr * 32 + lane, pair_bar = 1 + t * 4 + wr;
    if (work) {
      // The query rows of the CTA come by bulk copies to where converted values will lie, and are split in a rolled loop: 1200
      // instructions in a line, run once, took 14000 cycles, most of them to fetch the instructions.
      const uint32_t raw = w_ring;
      if (tid < PROMPT_ROWS) {
        const uint32_t x = x0 + tid, i = x / group, g = x - i * group;
        if (x < packed) {
          mbar_expect_tx(&raw_bar, DIM * 2);
          bulk_load_at(raw + tid * (DIM * 2), q + (long long)(r.x + (int)i) * q_stride + (long long)(head * group + g) * DIM, DIM * 2, &raw_bar);
        } else {
          mbar_arrive(&raw_bar);
        }
      }
      wait(&raw_bar, 0);
      constexpr int LANES = DIM / 8, AT_ONCE = 512 / LANES;
      const int chunk = tid % LANES;
#pragma unroll 1
      for (int x = tid / LANES; x < PROMPT_ROWS; x += 2 * AT_ONCE) {
        float f[2][8], scale[2];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          uint4 u4 = make_uint4(0u, 0u, 0u, 0u);
          if (x0 + x + p * AT_ONCE < packed)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(u4.x), "=r"(u4.y), "=r"(u4.z), "=r"(u4.w)
                         : "r"(raw + (x + p * AT_ONCE) * (DIM * 2) + chunk * 16) : "memory");
          unpack(u4, f[p], q);
        }
#pragma unroll
        for (int p = 0; p < 2; ++p) scale[p] = query_scale<DIM>(f[p]);
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          const int row_x = x + p * AT_ONCE;
          store_query<DIM, 2, false>(f[p], scale[p], q_base + (row_x >> 7) * PL::Q_TILE, row_x & 127, 128, chunk);
          if (chunk == 0) q_scale[row_x] = scale[p] * scale_log2;
        }
      }
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(&q_bar);
    }
    cta_sync(9, 512);                                  // the rows' scales
    const uint32_t t_s = tmem + t * 128 + ((uint32_t)(wr * 32) << 16), t_o = t_s + 256 + half * (DIM / 2);
    const uint32_t x = x0 + row;
    const int3 see = seen(mask, len - n_rows + query(x), len);
    const float qk = q_scale[row];
    const int my_nt = nt[t];
    // a tile inside [in_lo, in_hi) is seen by every row of the warp
    const int in_hi = seen(mask, len - n_rows + query(x0 + t * 128 + wr * 32), len).z;
    const int in_lo = seen(mask, len - n_rows + query(x0 + t * 128 + wr * 32 + 31), len).y;
    float ref = -CUDART_INF_F, high = -CUDART_INF_F, l = 0.f;      // reference of weights, sums and l; the highest one so far
    bool alive = true;                                 // the same in a warp and its partner, who share a barrier per tile
    for (int i = 0; alive && i < n_tiles; ++i) {
      const int sc = i % SC_ST;
      if (i >= my_nt) {                                // the other tile goes on
        wait(&sc_full[sc], i / SC_ST);
        if (!ok) break;
        if (lane == 0) mbar_arrive(&sc_empty[sc]);
        continue;
      }
      const int base = token0(i) + half * 64;
      wait(&sc_full[sc], i / SC_ST);
      wait(&s_bar[t], i);
      ctc_fence_after();
      float s[64];
      ctmem_ld32(t_s + half * 64, *reinterpret_cast<float (*)[32]>(s));
      ctmem_ld32(t_s + half * 64 + 32, *reinterpret_cast<float (*)[32]>(s + 32));
      ctmem_wait_ld();
      float top = -CUDART_INF_F;
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const int pg = (half * 64 + 16 * h) >> c.log_page;
        const float k = qk * page_scale[sc][0][pg], e = page_scale[sc][1][pg];
#pragma unroll
        for (int j = 16 * h; j < 16 * h + 16; j += 2) {
          const float2 v = fma2(make_float2(s[j], s[j + 1]), make_float2(k, k), make_float2(e, e));
          s[j] = v.x;
          s[j + 1] = v.y;
        }
      }
      if (base < in_lo || base + 64 > in_hi) {
        // a bit per token that the row sees (comparing 64 token indexes with the row's bounds cost a tenth of the kernel, in registers
        // of the tiles that need none of it)
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const uint32_t on = bits(see.y - base - 32 * w, see.z - base - 32 * w) | bits(0, see.x - base - 32 * w);
#pragma unroll
          for (int j = 0; j < 32; ++j) s[32 * w + j] = on & 1u << j ? s[32 * w + j] : -CUDART_INF_F;
        }
      }
#pragma unroll
      for (int j = 0; j < 64; j += 2) top = fmaxf(fmaxf(top, s[j]), s[j + 1]);
      half_s[half][row] = top;
      if (cta_sync_or(pair_bar, 64, !ok)) { alive = false; ok = false; break; }
      top = fmaxf(top, half_s[half ^ 1][row]);
      // the products of the tiles before are complete: scores of this one were issued behind them
      // (a tile that the row does not see moves nothing)
      const bool move = top > ref + 15.f || (top < ref - 5.f && top > -CUDART_INF_F);
      if (__any_sync(0xFFFFFFFFu, move)) {
        const float want = fmaxf(top - 7.f, high - 16.f);
        const float by = move ? ex2(ref - want) : 1.f;
        ref = move ? want : ref;
        high = fmaxf(high, ref);
        l *= by;
        if (i > 0 && __any_sync(0xFFFFFFFFu, by != 1.f)) {
#pragma unroll 1
          for (int cc = 0; cc < DIM / 2; cc += 16) {
            float o[16];
            ctmem_ld16(t_o + cc, o);
            ctmem_wait_ld();
            uint32_t w[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) w[j] = __float_as_uint(o[j] * by);
            ctmem_st16(t_o + cc, w);
          }
        }
      }
      const float m = ref == -CUDART_INF_F ? 0.f : -ref;
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const int pg = (half * 64 + 16 * h) >> c.log_page;
        float2 sum = make_float2(0.f, 0.f);
#pragma unroll
        for (int j = 16 * h; j < 16 * h + 16; j += 2) {
          float2 v = add2(make_float2(s[j], s[j + 1]), make_float2(m, m));
          v = make_float2(ex2(v.x), ex2(v.y));
          sum = add2(sum, v);
          s[j / 2] = __uint_as_float(to_f16x2(v.x, v.y));
        }
        l = fmaf(sum.x + sum.y, base + 16 * h < len ? page_scale[sc][2][pg] : 0.f, l);
      }
      ctmem_st32(t_s + half * 32, s);                  // (in the place of scores that both warps have read)
      ctmem_wait_st();
      ctc_fence_before();
      __syncwarp();
      if (lane == 0) { mbar_arrive(&p_bar[t]); mbar_arrive(&sc_empty[sc]); }
    }
    if (work && ok && my_nt > 0) wait(&o_bar[t], 0);
    half_s[half][row] = l;
    if (!cta_sync_or(pair_bar, 64, !ok) && work) {
      l += half_s[half ^ 1][row];
      const bool some = l > 0.f || l != l;
      const float inv = some ? 1.0f / l : 0.f;
      const uint32_t i = x / group, g = x - i * group;
      const long long at = (long long)(r.x + (int)i) * heads + head * group + g;
      if (x < packed && half == 0 && lse != nullptr) lse[at] = some ? (ref + log2f(l)) * 0.69314718055994531f : -CUDART_INF_F;
      ctc_fence_after();
      __nv_bfloat16* o_at = out + at * DIM + half * (DIM / 2);
#pragma unroll
      for (int cc = 0; cc < DIM / 2; cc += 32) {
        float o[32];
        ctmem_ld32(t_o + cc, o);
        ctmem_wait_ld();
        if (x < packed) {
#pragma unroll
          for (int j = 0; j < 32; j += 8) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = some ? pack_bf16x2(o[j + 2 * e] * inv, o[j + 2 * e + 1] * inv) : 0u;
            *reinterpret_cast<uint4*>(o_at + cc + j) = make_uint4(w[0], w[1], w[2], w[3]);
          }
        }
      }
    }
    if (!ok && lane == 0) atomicOr(status, STATUS_TIMEOUT);
  }
  ctc_fence_before();
  __syncthreads();
  if (warp == 19) tmem_free(tmem, 512);
}

}  // namespace ficoco
