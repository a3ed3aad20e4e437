// tcgen05 pieces shared by the tensor-core kernels of the 8-bit cache.
//
// The codes of the cache are operands as they lie in memory (kind::f8f6f4, e4m3 times e4m3, fp32 accumulation): nothing is
// converted on the way from HBM to the tensor cores.  What is not 8 bits wide, a query row or the softmax weights, is
// split instead: x = x0 + x1 / 16 + x2 / 256 + ..., each term the e4m3 value nearest to 16 times what the ones before it
// left.  A term leaves at most 2^-4 of its value, so two of them hold 8 significant bits (a bf16 value exactly), six
// hold 24.  Products of terms are exact in fp32.
#pragma once
#include <cuda.h>
#include "cache_common.cuh"

namespace ficoco {

constexpr int CTILE = 128;      // tokens per tile

__device__ __forceinline__ void ctc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void ctc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// Shared-memory descriptor of a tile whose rows are SWB bytes (128 or 64) under the swizzle of that width, eight-row groups
// one after the other.  The same for K-major operands (a row is an M or N index) and MN-major ones (a row is a K index).
template <int SWB>
__device__ __forceinline__ uint64_t cache_desc(uint32_t saddr) {
  uint64_t d = 0;
  d |= (uint64_t)((saddr & 0x3FFFFu) >> 4);
  d |= (uint64_t)1 << 16;                                // leading offset: no second swizzle row along it
  d |= (uint64_t)((8 * SWB) >> 4) << 32;                 // stride between eight-row groups
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)(SWB == 128 ? 2 : 4) << 61;
  return d;
}
// kind::f8f6f4: D fp32, A and B e4m3; a_mn / b_mn: that operand is MN-major.
__device__ __forceinline__ constexpr uint32_t cache_idesc(int m, int n, int a_mn, int b_mn) {
  return (1u << 4) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
// By a whole converged warp with uniform arguments; one elected lane issues.
__device__ __forceinline__ void mma_f8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "elect.sync _|q, 0xFFFFFFFF;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_commit(uint64_t* bar) {
  asm volatile(
      "{\n\t.reg .pred q;\n\t"
      "elect.sync _|q, 0xFFFFFFFF;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}"
      ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tmem_alloc(uint32_t* base_s, uint32_t cols) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(base_s)), "r"(cols) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t base, uint32_t cols) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(cols) : "memory");
}
__device__ __forceinline__ void ctmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// 16 accumulator columns of this thread's lane; complete at ctmem_wait_ld().
__device__ __forceinline__ void ctmem_ld16(uint32_t taddr, float* f) {
  uint32_t* r = reinterpret_cast<uint32_t*>(f);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr) : "memory");
}
// mbar_wait by a whole converged warp.  Every decision is a vote, so that the loop is a uniform one: lanes that leave a loop by
// themselves have to be brought together again, which costs more than the wait where the phase is complete.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, unsigned long long limit_ns) {
  const uint32_t a = smem_u32(bar);
  unsigned long long t0 = 0;
  for (;;) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.b32 %0, 1, 0, p;\n\t}"
        : "=r"(done) : "r"(a), "r"(parity) : "memory");
    if (__all_sync(0xFFFFFFFFu, done != 0)) return true;
    const unsigned long long t = sm_cycles();
    if (t0 == 0) t0 = t;
    else if (__any_sync(0xFFFFFFFFu, t - t0 > 2 * limit_ns)) return false;
  }
}
// An arrival that promises nothing about memory: for handing back what was only read (tensor memory behind its wait), by
// threads with global stores in flight.  The ordinary, releasing arrival waits for those, 900 cycles and more.
__device__ __forceinline__ void mbar_arrive_relaxed(uint64_t* bar) {
  asm volatile("mbarrier.arrive.relaxed.cta.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// Rows of codes, one box of page_size tokens, to shared memory in the swizzle that the tensor map names.
__device__ __forceinline__ void tma_rows(uint32_t dst, const CUtensorMap* map, int row, uint64_t* bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
               ::"r"(dst), "l"(map), "r"(0), "r"(row), "r"(smem_u32(bar)) : "memory");
}

// bulk_load to an address in shared memory.
__device__ __forceinline__ void bulk_load_at(uint32_t dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}

// A pair of values as NT e4m3 terms each: codes[t] holds both values' term t, the first one's in the low byte.  Term t is
// 16^t times what it stands for; with UP false the terms stand for themselves, so that products with all of them can share an
// accumulator (the smallest step of e4m3, 2^-9, then bounds all of them).
template <int NT, bool UP = true>
__device__ __forceinline__ void split_pair(float a, float b, uint32_t (&codes)[NT]) {
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    codes[t] = to_e4m3x2(a, b);
    if (t + 1 < NT) {
      const float2 got = from_e4m3x2(codes[t]);
      a = UP ? (a - got.x) * 16.f : a - got.x;
      b = UP ? (b - got.y) * 16.f : b - got.y;
    }
  }
}
__device__ __forceinline__ float2 mul2(const float2& a, const float2& b) {
  unsigned long long d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d)
      : "l"(reinterpret_cast<const unsigned long long&>(a)), "l"(reinterpret_cast<const unsigned long long&>(b)));
  return reinterpret_cast<const float2&>(d);
}
__device__ __forceinline__ float2 add2(const float2& a, const float2& b) {
  unsigned long long d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d)
      : "l"(reinterpret_cast<const unsigned long long&>(a)), "l"(reinterpret_cast<const unsigned long long&>(b)));
  return reinterpret_cast<const float2&>(d);
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float warp_max(float x) {
  float y;
  asm volatile("redux.sync.max.f32 %0, %1, 0xFFFFFFFF;" : "=f"(y) : "f"(x));
  return y;
}

// The rows of q of one item in shared memory as a K-major B or A operand: DIM bytes per row, row t * n_rows + r holds term t of
// row r, scaled by a power of two to at most 448.  Threads of `count` work on rows in groups of DIM / 8 lanes.
template <int DIM>
__device__ __forceinline__ uint32_t swizzled(int row, int chunk8) {       // byte offset of eight codes
  constexpr int XM = DIM == 128 ? 7 : 3;
  const int x = DIM == 128 ? row & 7 : (row >> 1) & 3;
  return (uint32_t)(row * DIM + ((((chunk8 >> 1) ^ x) & XM) << 4) + (chunk8 & 1) * 8);
}
__device__ __forceinline__ void st_shared8(uint32_t at, uint32_t lo, uint32_t hi) {
  asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at), "r"(lo), "r"(hi) : "memory");
}
__device__ __forceinline__ void st_shared1(uint32_t at, uint32_t byte) {
  asm volatile("st.shared.b8 [%0], %1;" ::"r"(at), "r"(byte) : "memory");
}
__device__ __forceinline__ void st_shared16(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// What a query row is divided by, a power of two that brings it to 448 at most (NaN where the row holds a NaN or an
// infinity), from the eight elements that each of its DIM / 8 lanes, neighbours in a warp, has.
template <int DIM>
__device__ __forceinline__ float query_scale(const float (&f)[8]) {
  uint32_t top = 0;                                      // order of magnitudes as integers: infinity and NaN are the largest
#pragma unroll
  for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(f[j]) & 0x7FFFFFFFu);
#pragma unroll
  for (int o = DIM / 16; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
  return top >= 0x7F800000u ? CUDART_NAN_F : scale_of(__uint_as_float(top));
}
// Those elements as NT terms, rows `rows` apart.
template <int DIM, int NT, bool UP = true>
__device__ __forceinline__ void store_query(const float (&f)[8], float scale, uint32_t base, int row, int rows, int chunk8) {
  const float inv = scale == scale ? 1.0f / scale : 0.f;
  uint32_t c[4][NT];
#pragma unroll
  for (int j = 0; j < 4; ++j) split_pair<NT, UP>(f[2 * j] * inv, f[2 * j + 1] * inv, c[j]);
#pragma unroll
  for (int t = 0; t < NT; ++t)
    st_shared8(base + swizzled<DIM>(t * rows + row, chunk8), c[0][t] | c[1][t] << 16, c[2][t] | c[3][t] << 16);
}

}  // namespace ficoco
