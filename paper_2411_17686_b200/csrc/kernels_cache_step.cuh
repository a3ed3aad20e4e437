// Attention over the 8-bit cache for few query rows per sequence (single tokens), on the 5th-generation tensor cores.
//
// Mathematics.  For a tile of 128 tokens and the RB query rows that share a key/value head, S^T = K Q^T and
// O^T = V^T P^T: the codes are operand A of both products (128 rows: tokens, then dimensions) as TMA brought them, the few
// query rows are the columns.  With s_j the score in units of log2 and e_j = log2 of the page's value scale, t_j = s_j + e_j
// and the weights are P_j = 2^(t_j - max), so that codes can be summed without their scale; the denominator sums P_j / 2^e_j.  Rows
// and weights are split into NT e4m3 terms (cache_umma.cuh), one more block of columns each.
//
// The maximum is that of 32 tokens: warp w works on tokens 32 w .. 32 w + 31 of every tile, which are one K step of the second
// product, so each step gets an accumulator of its own and the four are joined, with the factors that bring them to one
// maximum, where they are added to the fp32 sums in registers.  No barrier stands between a tile's scores and its weights.  The
// 8-bit terms end 2^-22 (six terms: 2^-38) below what they are relative to, so that a running maximum would lose the tokens behind
// a dominant one (a first token with nearly all of the weight and a value near zero: behind a score 16 above theirs the warp that had it lost
// all of its tokens, a quarter of the result); relative to 32 neighbours, of them alone.  The denominator, in fp32, keeps a running maximum per warp.
//
// What bounds it: HBM, one byte per key or value element.  The tensor cores are idle most of the time and nothing is
// converted, so an SM needs about 200 instructions per warp and tile of 32 KB.  All tiles of all (sequence, row block, head)
// items form one list which is cut into equal pieces, one per CTA (two CTAs per SM, so that one's softmax runs under the other's
// loads): ragged lengths balance by themselves.  An item that is cut leaves partial results; the CTA that finishes
// it last joins them in the order of the list, so the result does not depend on who that was.
//
// Roles: warps 0-3 softmax (thread = token of the tile), warps 4-7 queries and output (thread = dimension), warp 8 TMA and
// page scales, warp 9 MMA.  Tile i's scores are computed while tile i - 1's weights are multiplied; keys are given back as
// soon as the scores exist; queries are two items ahead, page indexes two and scales one batch of 32 / (pages per tile) tiles.
//
// Measured (bf16, heads of 128, replayed from a graph): 32 sequences of 4096 tokens and 8 heads 56 us, 4.8 TB/s; 64 ragged ones of 64 to 8192
// tokens 65 us, 3.3 TB/s; a window of 8000 tokens of 8 sequences 38 us; one sequence of 640 tokens and 32 heads 12.4 us; one tile 8.6 us, which
// is what start and end of a CTA take.  fp32 rows, one sequence of 65536 tokens: 54 us, 2.5 TB/s (45 with a maximum common to the four softmax
// warps, which costs bf16 rows a barrier per tile).
#pragma once
#include <float.h>
#include "cache_umma.cuh"

namespace ficoco {

constexpr int STEP_THREADS = 320;
constexpr int STEP_MAX_PARTS = 64;         // most pieces that an item is cut into

// One sequence of the call, in tiles.
struct StepSeq {
  int len, row0, n_rows, blocks, t_sink, t0, nt;
};
__device__ __forceinline__ StepSeq step_seq(const CacheView& c, const int* cu, int rows, int group, int rb, const MaskRule& mask,
                                            int b, unsigned* status) {
  StepSeq s;
  s.len = cache_length(c, b, status);
  const int2 r = cache_rows(cu, b, rows, status);
  s.row0 = r.x;
  s.n_rows = r.y - r.x;
  s.blocks = (int)(((uint32_t)s.n_rows * (uint32_t)group + rb - 1) / rb);
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
  int left;                                // tiles of the piece that are still to come
  int b, head, block, tile;
  StepSeq s;
};
__device__ __forceinline__ bool step_next(StepWalk& w, StepSeg& g, const CacheView& c, const int* cu, int rows, int group, int rb,
                                          const MaskRule& mask, unsigned* status) {
  if (w.left <= 0) return false;
  if (w.tile >= w.s.nt) {
    w.tile = 0;
    if (++w.head == c.kv) { w.head = 0; ++w.block; }
  }
  while (w.block >= w.s.blocks && w.b + 1 < c.batch) {
    w.block = 0;
    w.s = step_seq(c, cu, rows, group, rb, mask, ++w.b, status);
  }
  g.b = w.b; g.head = w.head; g.block = w.block; g.tile = w.tile; g.s = w.s;
  g.count = min(w.s.nt - w.tile, w.left);
  w.tile += g.count;
  w.left -= g.count;
  return true;
}
// The list of `total` tiles (below 2^31: the host sees to that) in n pieces, the first `more` of them a tile longer.
struct StepCut {
  int base, more;
  __device__ __forceinline__ StepCut(int total, int n) : base(total / n), more(total - total / n * n) {}
  __device__ __forceinline__ int start(int k) const { return k * base + min(k, more); }
  __device__ __forceinline__ int piece_of(int x) const {       // base > 0
    const int edge = more * (base + 1);
    return x < edge ? x / (base + 1) : more + (x - edge) / base;
  }
};
__device__ __forceinline__ int step_token0(const StepSeq& s, int tile) {      // first token of a tile of the item
  return (tile < s.t_sink ? tile : tile - s.t_sink + s.t0) * CTILE;
}

template <int DIM, int NT, int RB>
struct StepPlan {
  static constexpr int N = NT * RB;                                  // columns of both products
  static constexpr int HALF = CTILE * DIM;                           // keys or values of a tile
  static constexpr int Q_BYTES = (N * DIM + 1023) / 1024 * 1024, P_BYTES = N * CTILE;
  // half an SM's shared memory, less what is static: RB * DIM floats, 288 bytes per row and 768
  static constexpr int ROOM = 112 * 1024 - RB * (DIM * 4 + 288) - 768;
  static constexpr int STAGES_FIT = (ROOM - 1024 - 2 * (Q_BYTES + P_BYTES)) / (2 * HALF);
  static constexpr int STAGES = STAGES_FIT > 6 ? 6 : STAGES_FIT;
  static constexpr int SMEM = 1024 + STAGES * 2 * HALF + 2 * (Q_BYTES + P_BYTES);
  // 256 of the SM's 512 TMEM columns: score buffers of N and output buffers of 4 N columns
  static constexpr int NS = 10 * N <= 256 || 6 * N <= 256 ? 2 : 1, NO = 10 * N <= 256 ? 2 : 1;
  static constexpr int TMEM = 256;
  static constexpr int PART = RB * (DIM + 2);                        // floats of a partial result
  static_assert(STAGES >= 2 && (NS + 4 * NO) * N <= TMEM && N % 16 == 0, "two CTAs per SM");
};

// x[k] without a branch (any value for k >= RB).
template <int RB>
__device__ __forceinline__ float pick(const float (&x)[RB], int k) {
  float v = x[0];
#pragma unroll
  for (int r = 1; r < RB; ++r) v = k == r ? x[r] : v;
  return v;
}

// Sums of x[0 .. RB) over the warp; lane r (r < RB) gets that of x[r].  Halves the values that a lane holds with every
// exchange: RB - 1 shuffles and as many more as are left of the five steps, not five for each value.
template <int RB>
__device__ __forceinline__ float warp_sums(float (&x)[RB], int lane) {
#pragma unroll
  for (int bit = RB / 2; bit > 0; bit >>= 1) {
    const bool up = lane & bit;
#pragma unroll
    for (int r = 0; r < bit; ++r) {
      const float keep = up ? x[r + bit] : x[r], give = up ? x[r] : x[r + bit];
      x[r] = keep + __shfl_xor_sync(0xFFFFFFFFu, give, bit);
    }
  }
  float v = x[0];
#pragma unroll
  for (int bit = RB; bit < 32; bit <<= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, bit);
  return v;
}

// This thread's lane of the RB sums whose terms are NT blocks of RB accumulator columns, smallest term first.
template <int NT, int RB>
__device__ __forceinline__ void load_sums(uint32_t taddr, float (&x)[RB]) {
  static_assert(RB == 8 || RB == 16, "16 columns are two terms or one");
#pragma unroll
  for (int n = NT * RB - 16; n >= 0; n -= 16) {
    float f[16];
    ctmem_ld16(taddr + n, f);
    ctmem_wait_ld();
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      if (n + 16 == NT * RB) x[r] = f[16 - RB + r];
      else x[r] = fmaf(x[r], 0.0625f, f[16 - RB + r]);
      if (RB == 8) x[r] = fmaf(x[r], 0.0625f, f[r]);
    }
  }
}

template <class T, int DIM, int NT, int RB>
__global__ void __launch_bounds__(STEP_THREADS, 2) k_cache_step(
    const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap, const CacheView c,
    const T* __restrict__ q, const int* __restrict__ cu, T* __restrict__ out, float* __restrict__ lse, long long q_stride,
    float scale_log2, int rows, int heads, const MaskRule mask, int* __restrict__ counters, float* __restrict__ partials,
    unsigned* __restrict__ status, unsigned long long wait_ns, int extra_arrivals) {
  using PL = StepPlan<DIM, NT, RB>;
  constexpr int N = PL::N, NST = PL::STAGES, NS = PL::NS, NO = PL::NO;
  extern __shared__ unsigned char step_raw[];
  __shared__ uint64_t k_full[NST], v_full[NST], k_empty[NST], v_empty[NST], scale_bar[NST];
  __shared__ uint64_t q_bar[2], s_bar[2], s_free[2], p_bar[2], o_bar[2], free_bar[2], l_bar[2], drain_bar;
  __shared__ uint32_t tmem_s;
  __shared__ float page_scale[NST][3][8];              // key scale, log2 of the value scale, 1 / value scale
  __shared__ float wmax[2][4][RB];                     // a tile's maxima per softmax warp, which its weights are relative to
  __shared__ __align__(16) float factor[2][4][5][RB];  // per output warp: what brings the four warps' sums, and the old ones, to one maximum
  __shared__ float l_s[2][4][RB], m_s[2][4][RB];       // denominators of an item per softmax warp, and the maxima that they are relative to
  __shared__ float q_scale[2][RB];
  __shared__ int2 row_see[2][RB];                      // tokens [x, y) of a row (and its sinks)
  __shared__ StepSeg seg_s[4];                         // the output warps' items: this one and the two ahead
  __shared__ __align__(16) float out_s[RB][DIM];       // an item's sums
  __shared__ float top_s[RB], den_s[RB];               // its maxima and denominators
  __shared__ int last_s, dead_s;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t ring = (smem_u32(step_raw) + 1023u) & ~1023u;         // keys of all stages, then values
  const uint32_t v_ring = ring + NST * PL::HALF, q_base = v_ring + NST * PL::HALF, p_base = q_base + 2 * PL::Q_BYTES;
  const int group = heads / c.kv;
  if (tid == 0) {
    for (int s = 0; s < NST; ++s) {
      mbar_init(&k_full[s], 1); mbar_init(&v_full[s], 1); mbar_init(&k_empty[s], 1); mbar_init(&v_empty[s], 1);
      mbar_init(&scale_bar[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&q_bar[s], 128); mbar_init(&s_bar[s], 1); mbar_init(&s_free[s], 4); mbar_init(&p_bar[s], 4 + extra_arrivals);
      mbar_init(&o_bar[s], 1); mbar_init(&free_bar[s], 4); mbar_init(&l_bar[s], 4);
    }
    mbar_init(&drain_bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 9) tmem_alloc(&tmem_s, PL::TMEM);
  grid_dep_wait();
  // (one thread's look for the CTA: another CTA may raise the bit at any time)
  if (tid == 0) dead_s = (*reinterpret_cast<const volatile unsigned*>(status) & STATUS_TIMEOUT) ? 1 : 0;
  // ---- this CTA's piece of the list.  Every warp finds it by itself (lane = sequence), so that no barrier is waited for ------
  StepWalk walk;
  int total = 0, n_cta, piece0;
  {
    int nt_most = 0, size = 0;
    long long sum = 0;
    StepSeq s0;
#pragma unroll 1
    for (int b0 = 0; b0 < c.batch; b0 += 32) {
      size = 0;
      if (b0 + lane < c.batch) {
        s0 = step_seq(c, cu, rows, group, RB, mask, b0 + lane, status);
        size = s0.blocks * c.kv * s0.nt;
        if (size > 0) nt_most = max(nt_most, s0.nt);
      }
      sum += size;
    }
    // The host keeps the list below 2^31 tiles for sequences that share no row.  Offsets that go back to rows of earlier sequences can
    // make it longer: no place in it could be trusted then.
    if (__reduce_add_sync(0xFFFFFFFFu, (uint32_t)min(sum >> 16, 1ll << 26)) >= (1u << 15) - 32) {
      if (lane == 0) atomicOr(status, STATUS_CACHE);
      sum = 0;
      nt_most = 0;
    }
    total = __reduce_add_sync(0xFFFFFFFFu, (int)sum);
    nt_most = __reduce_max_sync(0xFFFFFFFFu, nt_most);
    // CTAs that get a piece: no more than tiles, nor so many that the longest item would be cut into more than STEP_MAX_PARTS
    n_cta = max(1, min((int)gridDim.x, total));
    const float most = (float)(STEP_MAX_PARTS - 2) * (float)total;
    if ((float)n_cta * (float)nt_most > most) n_cta = max(1, (int)(most / (float)nt_most));
    const StepCut cut(total, n_cta);
    piece0 = cut.start(blockIdx.x);
    walk.left = (int)blockIdx.x < n_cta ? cut.start(blockIdx.x + 1) - piece0 : 0;
    walk.b = 0; walk.head = walk.block = walk.tile = 0;
    if (walk.left > 0) {
      int before = 0;
#pragma unroll 1
      for (int b0 = 0;; b0 += 32) {
        if (c.batch > 32) {                                    // (the last 32 sequences' sizes are at hand)
          size = 0;
          if (b0 + lane < c.batch) {
            s0 = step_seq(c, cu, rows, group, RB, mask, b0 + lane, status);
            size = s0.blocks * c.kv * s0.nt;
          }
        }
        int upto = size;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int v = __shfl_up_sync(0xFFFFFFFFu, upto, o);
          upto += lane >= o ? v : 0;
        }
        const unsigned reached = __ballot_sync(0xFFFFFFFFu, before + upto > piece0);
        if (reached == 0 && b0 + 32 < c.batch) {
          before += __shfl_sync(0xFFFFFFFFu, upto, 31);
          continue;
        }
        const int l = reached ? __ffs(reached) - 1 : 31;
        walk.b = b0 + l;
        walk.s.len = __shfl_sync(0xFFFFFFFFu, s0.len, l); walk.s.row0 = __shfl_sync(0xFFFFFFFFu, s0.row0, l);
        walk.s.n_rows = __shfl_sync(0xFFFFFFFFu, s0.n_rows, l); walk.s.blocks = __shfl_sync(0xFFFFFFFFu, s0.blocks, l);
        walk.s.t_sink = __shfl_sync(0xFFFFFFFFu, s0.t_sink, l); walk.s.t0 = __shfl_sync(0xFFFFFFFFu, s0.t0, l);
        walk.s.nt = __shfl_sync(0xFFFFFFFFu, s0.nt, l);
        const uint32_t off = (uint32_t)(piece0 - before - __shfl_sync(0xFFFFFFFFu, upto - size, l));
        const uint32_t item = off / (uint32_t)walk.s.nt;
        walk.tile = (int)(off - item * (uint32_t)walk.s.nt);
        walk.block = (int)(item / (uint32_t)c.kv);
        walk.head = (int)item - walk.block * c.kv;
        break;
      }
    }
  }
  ctc_fence_before();
  __syncthreads();                                             // barriers, TMEM
  ctc_fence_after();
  grid_dep_launch();       // behind the barrier: a dependent that took this CTA's TMEM first would wait for it for ever
  const uint32_t tmem = tmem_s;
  if (dead_s) walk.left = 0;
  bool ok = true;                                      // the same in all lanes of a warp
  auto wait = [&](uint64_t* bar, int phase) { ok = ok && warp_wait(bar, (uint32_t)phase & 1u, wait_ns); };

  if (warp == 8) {
    // ---------------- TMA.  Lane = (tile of a batch, page of the tile) -------------------------------------------------------
    const int log_ppt = 7 - c.log_page, ppt = 1 << log_ppt, batch_tiles = 32 >> log_ppt, my_page = lane & (ppt - 1);
    StepSeg g;
    int t_next = 0, t_end = 0;
    struct Batch { int page, head, tiles; float ks, vs; };
    // The next batch: this lane's page (-1: none) and head, tiles in the batch.
    auto assign = [&](Batch& x, int most) {
      x.page = -1;
      x.ks = x.vs = 1.f;
      int b = 0, base = 0, len = 0;
#pragma unroll 1
      for (x.tiles = 0; x.tiles < most; ++x.tiles, ++t_next) {
        if (t_next >= t_end) {
          if (!step_next(walk, g, c, cu, rows, group, RB, mask, status)) break;
          t_next = g.tile;
          t_end = g.tile + g.count;
        }
        const bool on = lane >> log_ppt == x.tiles;            // (a branch that some lanes take costs 160 cycles)
        b = on ? g.b : b;
        base = on ? step_token0(g.s, t_next) : base;
        len = on ? g.s.len : len;
        x.head = on ? g.head : x.head;
      }
      base += my_page << c.log_page;
      if (base < len) x.page = cache_page(c, b, base >> c.log_page, 0, status);
    };
    auto fetch_scales = [&](Batch& x) {
      if (x.page >= 0) {
        const size_t at = (size_t)x.page * c.kv + x.head;
        x.ks = c.ks[at];
        x.vs = c.vs[at];
      }
    };
    Batch now, soon, later;
    now.head = soon.head = later.head = 0;
    assign(now, min(batch_tiles, NST));
    fetch_scales(now);
    const uint32_t bytes = (uint32_t)(c.page * DIM);
    int i = 0, st = 0, wrap = -1, st_before = 0;
    float v3[3];                                         // scales of the tile before this one, whose turn is one tile late:
    bool held = false;                                   // the first batch's are still on their way when its copies go out
    auto deliver = [&]() {
      if (held) {
#pragma unroll
        for (int x = 0; x < 3; ++x) page_scale[st_before][x][my_page] = v3[x];
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&scale_bar[st_before]);
    };
    bool first = true;
#pragma unroll 1
    while (ok && now.tiles > 0) {
      if (!first) { fetch_scales(soon); assign(later, batch_tiles); }
#pragma unroll 1
      for (int t = 0; t < now.tiles; ++t, ++i) {
        const bool mine_now = lane >> log_ppt == t && now.page >= 0;
        const uint32_t load = bytes * (uint32_t)__popc(__ballot_sync(0xFFFFFFFFu, mine_now));
        const uint32_t dst = ring + (uint32_t)st * PL::HALF + (uint32_t)my_page * bytes;
        const int row = (now.page * c.kv + now.head) << c.log_page;
        if (i >= NST) wait(&k_empty[st], wrap);
        if (ok) {
          if (lane == 0) mbar_expect_tx(&k_full[st], load);
          __syncwarp();
          if (mine_now) tma_rows(dst, &kmap, row, &k_full[st]);
          if (i >= NST) wait(&v_empty[st], wrap);
          if (!ok && lane == 0) mbar_wait(&k_full[st], (uint32_t)(wrap + 1) & 1u, wait_ns);
        }
        if (!ok) break;
        if (lane == 0) mbar_expect_tx(&v_full[st], load);
        __syncwarp();
        if (mine_now) tma_rows(dst + NST * PL::HALF, &vmap, row, &v_full[st]);
        if (i > 0) deliver();
        held = mine_now;
        if (mine_now) { v3[0] = now.ks; v3[1] = log2f(now.vs); v3[2] = 1.0f / now.vs; }
        st_before = st;
        if (++st == NST) { st = 0; ++wrap; }
        if (first && t + 1 == now.tiles) {                     // the ring is full: time for the batches behind
          first = false;
          assign(soon, batch_tiles);
          fetch_scales(soon);
          assign(later, batch_tiles);
        }
      }
      now = soon;
      soon = later;
    }
    if (i > 0 && ok) deliver();
    if (!ok) {
      if (lane == 0) atomicOr(status, STATUS_TIMEOUT);
      // no copy outlives the CTA: the tiles asked for last
#pragma unroll 1
      for (int k = max(0, i - NST); k < i; ++k) {
        mbar_wait(&k_full[k % NST], (k / NST) & 1, wait_ns);
        mbar_wait(&v_full[k % NST], (k / NST) & 1, wait_ns);
      }
    }
  } else if (warp == 9) {
    // ---------------- MMA: scores of tile i go out before the weights of tile i - 1 are waited for ------------------------
    const uint32_t u_tmem = __shfl_sync(0xFFFFFFFFu, tmem, 0);
    constexpr uint32_t id_s = cache_idesc(128, N, 0, 0), id_o = cache_idesc(DIM, N, 1, 0);
    StepSeg g;
    int seg = -1, left = 0, st = 0, wrap = 0, st_prev = 0, wrap_prev = 0;
#pragma unroll 1
    for (int i = 0;; ++i) {
      bool more = true;
      if (left == 0) {
        more = step_next(walk, g, c, cu, rows, group, RB, mask, status);
        if (more) {
          ++seg;
          left = g.count;
          wait(&q_bar[seg & 1], seg >> 1);
        }
      }
      if (more) {
        --left;
        wait(&k_full[st], wrap);
        if (i >= NS) wait(&s_free[i % NS], (i / NS) - 1);
        if (!ok) break;
        ctc_fence_after();
        const uint64_t ad = cache_desc<DIM>(ring + (uint32_t)st * PL::HALF);
        const uint64_t bd = cache_desc<DIM>(q_base + (uint32_t)(seg & 1) * PL::Q_BYTES);
#pragma unroll
        for (int k = 0; k < DIM / 32; ++k) mma_f8(u_tmem + (uint32_t)(i % NS) * N, ad + 2 * k, bd + 2 * k, id_s, k > 0);
        mma_commit(&s_bar[i % NS]);
        mma_commit(&k_empty[st]);
      }
      if (i > 0) {
        const int j = i - 1;
        wait(&v_full[st_prev], wrap_prev);
        wait(&p_bar[j & 1], j >> 1);
        if (NO == 1 && j > 0) wait(&free_bar[(j - 1) & 1], (j - 1) >> 1);
        if (!ok) break;
        ctc_fence_after();
        const uint64_t ad = cache_desc<DIM>(v_ring + (uint32_t)st_prev * PL::HALF);
        const uint64_t bd = cache_desc<128>(p_base + (uint32_t)(j & 1) * PL::P_BYTES);
#pragma unroll
        for (int k = 0; k < 4; ++k)      // a softmax warp's tokens each, into columns of its own
          mma_f8(u_tmem + NS * N + (uint32_t)((j % NO) * 4 + k) * N, ad + (uint64_t)(k * (32 * DIM >> 4)), bd + 2 * k, id_o, 0);
        mma_commit(&o_bar[j % NO]);
        mma_commit(&v_empty[st_prev]);
      }
      if (!more) break;
      st_prev = st;
      wrap_prev = wrap;
      if (++st == NST) { st = 0; ++wrap; }
    }
    if (!ok) {
      if (lane == 0) atomicOr(status, STATUS_TIMEOUT);
      mma_commit(&drain_bar);
      mbar_wait(&drain_bar, 0, wait_ns);
    }
  } else if (warp < 4) {
    // ---------------- softmax: thread = token of the tile; the warps go their own ways ------------------------------------
    const uint32_t t_lane = tmem + ((uint32_t)(warp * 32) << 16);
    StepSeg g;
    int i = 0, st = 0, wrap = 0;
    const int pg = tid >> c.log_page;
#pragma unroll 1
    for (int seg = 0; ok && step_next(walk, g, c, cu, rows, group, RB, mask, status); ++seg) {
      const int buf_q = seg & 1;
      wait(&q_bar[buf_q], seg >> 1);                           // the rows' scales and masks
      float m[RB], l[RB];                                      // the warp's largest so far, the denominators relative to it
#pragma unroll
      for (int r = 0; r < RB; ++r) { m[r] = -FLT_MAX; l[r] = 0.f; }
      // a tile inside [in_lo, in_hi) is seen by every row of the item
      const int i_first = (int)((uint32_t)g.block * RB / (uint32_t)group);
      const int i_last = min((int)(((uint32_t)g.block * RB + RB - 1) / (uint32_t)group), g.s.n_rows - 1);
      const int in_hi = seen(mask, g.s.len - g.s.n_rows + i_first, g.s.len).z;
      const int in_lo = seen(mask, g.s.len - g.s.n_rows + i_last, g.s.len).y;
#pragma unroll 1
      for (int t = g.tile; t < g.tile + g.count; ++t, ++i) {
        const int base = step_token0(g.s, t), buf = i & 1;
        wait(&scale_bar[st], wrap);
        const bool token = base + tid < g.s.len;               // (pages behind the last one have no scales)
        const float ks = page_scale[st][0][pg], ve = page_scale[st][1][pg], vi = token ? page_scale[st][2][pg] : 0.f;
        wait(&s_bar[i % NS], i / NS);
        if (!ok) break;
        ctc_fence_after();
        float s[RB];
        load_sums<NT, RB>(t_lane + (uint32_t)(i % NS) * N, s);
        ctc_fence_before();
        if (lane == 0) mbar_arrive(&s_free[i % NS]);
        const bool edge = base < in_lo || base + CTILE > in_hi;
#pragma unroll
        for (int r = 0; r < RB; ++r) s[r] = fmaf(s[r], q_scale[buf_q][r] * ks, ve);
        if (edge) {
          const int j = base + tid;
#pragma unroll
          for (int r = 0; r < RB; ++r) {
            const int2 see = row_see[buf_q][r];
            const bool on = j < see.y && (j >= see.x || j < mask.sinks);
            s[r] = on ? s[r] : -CUDART_INF_F;
          }
          if (base + CTILE > g.s.len) {                        // no token: whatever the slot holds must not meet a weight of 0
            wait(&v_full[st], wrap);
            if (!ok) break;
            if (!token) {
              const uint32_t v = v_ring + (uint32_t)st * PL::HALF + tid * DIM;
#pragma unroll
              for (int x = 0; x < DIM; x += 16) st_shared16(v + x, 0u, 0u, 0u, 0u);
            }
          }
        }
        float top[RB];                                         // of these 32 tokens (-FLT_MAX: none is seen)
#pragma unroll
        for (int r = 0; r < RB; ++r) {
          top[r] = fmaxf(warp_max(s[r]), -FLT_MAX);
          s[r] = ex2(s[r] - top[r]);
          // old sum and new weight brought to the larger of the two maxima: one of the factors is 1
          const float d = m[r] - top[r], e = ex2(-fabsf(d)), w = s[r] * vi;
          l[r] = d > 0.f ? fmaf(w, e, l[r]) : fmaf(l[r], e, w);
          m[r] = fmaxf(m[r], top[r]);
        }
        if (i >= 2) wait(&free_bar[buf], (i >> 1) - 1);        // the weights and maxima of tile i - 2 have been used
        if (!ok) break;
        {                                                      // (a store per row under `lane == r` took 160 cycles each)
          const float mine_m = pick<RB>(top, lane);
          if (lane < RB) wmax[buf][warp][lane] = mine_m;
        }
        const uint32_t p = p_base + (uint32_t)buf * PL::P_BYTES + (tid & 15);
#pragma unroll
        for (int r = 0; r < RB; r += 2) {
          uint32_t code[NT];
          split_pair<NT>(s[r] * 256.f, s[r + 1] * 256.f, code);
#pragma unroll
          for (int u = 0; u < NT; ++u) {
            const int n = u * RB + r;
            st_shared1(p + n * 128 + ((((tid >> 4) ^ n) & 7) << 4), code[u] & 0xFFu);
            st_shared1(p + (n + 1) * 128 + ((((tid >> 4) ^ (n + 1)) & 7) << 4), code[u] >> 8);
          }
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_bar[buf]);
        if (++st == NST) { st = 0; ++wrap; }
      }
      if (!ok) break;
      const float mine_m = pick<RB>(m, lane), sum = warp_sums<RB>(l, lane);
      if (lane < RB) { l_s[buf_q][warp][lane] = sum; m_s[buf_q][warp][lane] = mine_m; }
      __syncwarp();
      if (lane == 0) mbar_arrive(&l_bar[buf_q]);
    }
    if (!ok && lane == 0) atomicOr(status, STATUS_TIMEOUT);
  } else {
    // ---------------- queries and output: thread = dimension -------------------------------------------------------------
    const int bt = tid - 128, bw = warp - 4;
    const uint32_t t_lane = tmem + ((uint32_t)(bw * 32) << 16);
    constexpr int LANES = DIM / 8, PASS_ROWS = 128 / LANES, PASSES = (RB + PASS_ROWS - 1) / PASS_ROWS;
    const int q_chunk = bt % LANES, q_row = bt / LANES;
    Raw8<T> qf[PASSES];
    // rows of an item: row x of block k is head x % group of the sequence's row x / group
    auto load_q = [&](const StepSeg& g) {
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        const uint32_t x = (uint32_t)g.block * RB + p * PASS_ROWS + q_row;
        const int i = (int)(x / (uint32_t)group), h = g.head * group + (int)(x - (uint32_t)i * group);
        const bool on = p * PASS_ROWS + q_row < RB && i < g.s.n_rows;
        if (on) qf[p].load(q + (long long)(g.s.row0 + i) * q_stride + (long long)h * DIM + q_chunk * 8);
        else qf[p].clear();
      }
    };
    auto put_q = [&](const StepSeg& g, int buf) {
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        const int r = p * PASS_ROWS + q_row;
        if (PASSES * PASS_ROWS > RB && r >= RB) continue;      // (whole warps: RB is a multiple of a warp's rows)
        float f[8];
        qf[p].get(f);
        const float s = query_scale<DIM>(f);
        store_query<DIM, NT>(f, s, q_base + (uint32_t)buf * PL::Q_BYTES, r, RB, q_chunk);
        if (q_chunk == 0) q_scale[buf][r] = s * scale_log2;
      }
      if (bt < RB) {
        const uint32_t x = (uint32_t)g.block * RB + bt;
        const int i = min((int)(x / (uint32_t)group), g.s.n_rows);
        const int3 see = seen(mask, g.s.len - g.s.n_rows + i, g.s.len);
        row_see[buf][bt] = i < g.s.n_rows ? make_int2(see.y, see.z) : make_int2(0, 0);
      }
      fence_proxy_async();
      mbar_arrive(&q_bar[buf]);
    };
    // item k's description goes to seg_s[k % 4]; returns whether there is one, its query rows asked for
    auto ahead = [&](int k) {
      StepSeg g;
      if (!step_next(walk, g, c, cu, rows, group, RB, mask, status)) return false;
      load_q(g);
      if (bt == 0) seg_s[k & 3] = g;
      return true;
    };
    int at = piece0;                                           // where this item's tiles start in the list
    int n_seg = 0;                                             // items described so far
    bool more = true;
    int i = 0;
    constexpr int PER = RB / 8;                                // maxima per lane: lane = (softmax warp, row % 8)
    // Three turns ahead of item 0 only fetch and place queries: the code stands here once (all of a kernel's roles share the
    // instruction caches, and what is fetched for the first time takes longer than what it does).
#pragma unroll 1
    for (int seg = -3; seg < n_seg; ++seg) {
      if (seg < 0) {
        cta_sync(2, 128);                                      // the items' descriptions
        if (seg + 2 >= 0 && seg + 2 < n_seg) put_q(seg_s[seg + 2], seg & 1);
        if (more) {
          more = ahead(n_seg);
          n_seg += more;
        }
        if (n_seg == 0) break;
        continue;
      }
      const int buf_q = seg & 1;
      const StepSeg& g = seg_s[seg & 3];
      const int count = g.count;
      float acc[RB], m_run[PER];
#pragma unroll
      for (int r = 0; r < RB; ++r) acc[r] = 0.f;
#pragma unroll
      for (int p = 0; p < PER; ++p) m_run[p] = -FLT_MAX;
#pragma unroll 1
      for (int t = 1; t <= count; ++t, ++i) {
        const int buf = i & 1;
        wait(&p_bar[buf], i >> 1);                             // the maxima
        float (*f)[RB] = factor[buf][bw];
#pragma unroll
        for (int p = 0; p < PER; ++p) {
          const int w = lane >> 3, r = (lane & 7) + 8 * p;
          const float mw = wmax[buf][w][r];
          float mn = fmaxf(m_run[p], mw);
          mn = fmaxf(mn, __shfl_xor_sync(0xFFFFFFFFu, mn, 8));
          mn = fmaxf(mn, __shfl_xor_sync(0xFFFFFFFFu, mn, 16));
          f[w][r] = ex2(mw - mn);
          f[4][r] = ex2(m_run[p] - mn);                          // (the same from four lanes)
          m_run[p] = mn;
        }
        __syncwarp();
        wait(&o_bar[i % NO], i / NO);
        ctc_fence_after();
#pragma unroll
        for (int r = 0; r < RB; ++r) acc[r] *= f[4][r];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          float o[RB];
          load_sums<NT, RB>(t_lane + NS * N + (uint32_t)((i % NO) * 4 + w) * N, o);
#pragma unroll
          for (int r = 0; r < RB; ++r) acc[r] = fmaf(o[r], f[w][r], acc[r]);
        }
        ctc_fence_before();
        __syncwarp();
        if (t < count && lane == 0) mbar_arrive(&free_bar[buf]);
      }
      wait(&l_bar[buf_q], seg >> 1);
      cta_sync(2, 128);                                        // the item before this one has been read
      // (M = 64 accumulators lie in the first sixteen lanes of each warp)
      if (DIM == 128 || lane < 16) {
        const int d = DIM == 128 ? bt : bw * 16 + lane;
#pragma unroll
        for (int r = 0; r < RB; ++r) out_s[r][d] = acc[r];
      }
      if (bw == 0 && lane < RB) {
        const float top = lane < 8 ? m_run[0] : m_run[PER - 1];      // (the largest of m_s)
        float den = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) den = fmaf(l_s[buf_q][w][lane], ex2(m_s[buf_q][w][lane] - top), den);
        den_s[lane] = den;
        top_s[lane] = top;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&free_bar[(i - 1) & 1]);
      if (cta_sync_or(2, 128, !ok)) { ok = false; break; }     // one wait that ran out ends it for all 128 threads
      if (seg + 2 < n_seg) put_q(seg_s[(seg + 2) & 3], buf_q); // (every score of this item is computed and used)
      if (more) {
        more = ahead(n_seg);
        n_seg += more;
      }
      // Four dimensions of a row per thread and turn (rolled loops: an item's end runs few times, and code that is fetched for the
      // first time takes longer than what it does).
      const uint32_t x0 = (uint32_t)g.block * RB;
      const int nr = min(RB, (int)((uint32_t)g.s.n_rows * group - x0));
      auto place = [&](int r) {                                // where row r of the item lies in out and lse
        const uint32_t ri = (x0 + r) / (uint32_t)group;
        return (long long)(g.s.row0 + (int)ri) * heads + g.head * group + (int)(x0 + r - ri * group);
      };
      auto finish = [&](int r, int d4, const float4& v, float top, float den) {
        const bool some = den > 0.f || den != den;
        const float inv = some ? __fdividef(0.00390625f, den) : 0.f;
        const long long o_at = place(r);
        store4(out + o_at * DIM + d4, make_float4(some ? v.x * inv : 0.f, some ? v.y * inv : 0.f, some ? v.z * inv : 0.f, some ? v.w * inv : 0.f));
        if (lse != nullptr && d4 == 0) lse[o_at] = some ? (top + log2f(den)) * 0.69314718055994531f : -CUDART_INF_F;
      };
      if (count == g.s.nt) {
#pragma unroll 1
        for (int u = bt; u < nr * (DIM / 4); u += 128) {
          const int r = u / (DIM / 4), d4 = (u % (DIM / 4)) * 4;
          finish(r, d4, *reinterpret_cast<const float4*>(&out_s[r][d4]), top_s[r], den_s[r]);
        }
      } else {
        // A cut item.  Its first piece is the last one of CTA `owner`, the others are the first ones of the CTAs behind it.
        float* mine_p = partials + ((size_t)blockIdx.x * 2 + (g.tile == 0 ? 1 : 0)) * PL::PART;
#pragma unroll 1
        for (int u = bt; u < nr * (DIM / 4); u += 128)
          __stcg(reinterpret_cast<float4*>(mine_p + u * 4), *reinterpret_cast<const float4*>(&out_s[0][0] + u * 4));
        if (bt < nr) { __stcg(mine_p + RB * DIM + bt, top_s[bt]); __stcg(mine_p + RB * DIM + RB + bt, den_s[bt]); }
        const StepCut cut(total, n_cta);
        const int owner = cut.piece_of(at - g.tile), parts = cut.piece_of(at - g.tile + g.s.nt - 1) - owner + 1;
        cta_sync(2, 128);
        if (bt == 0) last_s = atom_acq_rel_add(&counters[owner], 1) == parts - 1;
        cta_sync(2, 128);
        if (last_s) {
          if (bt == 0) counters[owner] = 0;
          auto part = [&](int k) { return partials + ((size_t)(owner + k) * 2 + (k == 0 ? 1 : 0)) * PL::PART; };
#pragma unroll 1
          for (int u = bt; u < nr * (DIM / 4); u += 128) {
            const int r = u / (DIM / 4), d4 = (u % (DIM / 4)) * 4;
            float top = -FLT_MAX, den = 0.f;
            float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
            // eight parts at a time, in order, the sums brought to the larger maximum
#pragma unroll 1
            for (int k0 = 0; k0 < parts; k0 += 8) {
              float m8[8], l8[8];
              float4 v8[8];
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                const float* pk = part(min(k0 + k, parts - 1));
                m8[k] = __ldcg(pk + RB * DIM + r);
                l8[k] = __ldcg(pk + RB * DIM + RB + r);
                v8[k] = __ldcg(reinterpret_cast<const float4*>(pk + r * DIM + d4));
              }
              float mn = top;
#pragma unroll
              for (int k = 0; k < 8; ++k) mn = fmaxf(mn, m8[k]);       // (the last part again in the places behind it)
              const float w0 = ex2(top - mn);
              top = mn;
              den *= w0; a.x *= w0; a.y *= w0; a.z *= w0; a.w *= w0;
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                if (k0 + k >= parts) break;
                const float w = ex2(m8[k] - mn);
                den = fmaf(w, l8[k], den);
                a.x = fmaf(w, v8[k].x, a.x); a.y = fmaf(w, v8[k].y, a.y); a.z = fmaf(w, v8[k].z, a.z); a.w = fmaf(w, v8[k].w, a.w);
              }
            }
            finish(r, d4, a, top, den);
          }
        }
      }
      at += count;
    }
    if (!ok && lane == 0) atomicOr(status, STATUS_TIMEOUT);
  }
  ctc_fence_before();
  __syncthreads();
  if (warp == 9) tmem_free(tmem, PL::TMEM);
}

}  // namespace ficoco
