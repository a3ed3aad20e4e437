// Entry points of the 8-bit paged cache (ficoco.h: append, attention, weights, copy, compact) and the host's page pool.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <functional>
#include <initializer_list>
#include <new>
#include <queue>
#include <vector>

#include "../../include/ficoco.h"
#include "cache_common.cuh"
#include "ctx_access.h"
#include "kernels_cache_pages.cuh"
#include "kernels_cache_prompt.cuh"
#include "kernels_cache_simt.cuh"
#include "kernels_cache_step.cuh"
#include "kernels_cache_weights.cuh"

using namespace ficoco;

namespace {

template <class... KArgs, class... Args>
cudaError_t launch(void (*kernel)(KArgs...), dim3 grid, int block, size_t smem, cudaStream_t st, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...);
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
bool aligned4(const void* p) { return ((uintptr_t)p & 3) == 0; }
// Bytes that a call reads or writes (p NULL: none).
struct Span {
  const void* p;
  size_t n;
};
bool overlap(const Span& a, const Span& b) {
  const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
  return a.p && b.p && x < y + b.n && y < x + a.n;
}
bool overlap(std::initializer_list<Span> a, std::initializer_list<Span> b) {
  for (const Span& x : a)
    for (const Span& y : b)
      if (overlap(x, y)) return true;
  return false;
}

int check_cache(const ficoco_cache* c, CacheView* v) {
  if (!c || !c->k_codes || !c->v_codes || !c->k_scale || !c->v_scale || !c->page_table || !c->lengths) return FICOCO_ERR_INVALID_ARG;
  if (c->n_pages < 1 || c->kv_heads < 1 || c->head_dim < 1 || c->batch < 1 || c->max_pages < 1) return FICOCO_ERR_INVALID_ARG;
  if (c->table_stride < c->max_pages) return FICOCO_ERR_INVALID_ARG;
  if (!aligned16(c->k_codes) || !aligned16(c->v_codes)) return FICOCO_ERR_INVALID_ARG;
  if (!aligned4(c->k_scale) || !aligned4(c->v_scale) || !aligned4(c->page_table) || !aligned4(c->lengths)) return FICOCO_ERR_INVALID_ARG;
  if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128) return FICOCO_ERR_UNSUPPORTED;
  if (c->head_dim % 16 != 0 || c->head_dim > 256 || c->kv_heads > 1024 || c->batch > 65535) return FICOCO_ERR_UNSUPPORTED;
  if ((long long)c->n_pages * c->kv_heads * c->page_size > INT32_MAX) return FICOCO_ERR_UNSUPPORTED;   // rows of a tensor map
  if ((long long)c->max_pages * c->page_size > 1 << 30) return FICOCO_ERR_UNSUPPORTED;                 // tokens of a sequence
  v->k = (uint8_t*)c->k_codes; v->v = (uint8_t*)c->v_codes; v->ks = c->k_scale; v->vs = c->v_scale;
  v->table = c->page_table; v->len = c->lengths; v->table_stride = c->table_stride;
  v->n_pages = c->n_pages; v->page = c->page_size; v->kv = c->kv_heads; v->dim = c->head_dim;
  v->batch = c->batch; v->max_pages = c->max_pages;
  v->log_page = c->page_size == 16 ? 4 : c->page_size == 32 ? 5 : c->page_size == 64 ? 6 : 7;
  return FICOCO_OK;
}

// Rows of a call: pointer (none where there are no rows), stride, element type.
int check_rows(const void* p, int rows, long long stride, int dtype, long long row_elems) {
  if (rows < 0 || (rows > 0 && !p) || !aligned16(p) || stride < row_elems) return FICOCO_ERR_INVALID_ARG;
  if (dtype != FICOCO_FP32 && dtype != FICOCO_BF16) return FICOCO_ERR_UNSUPPORTED;
  const int es = dtype == FICOCO_BF16 ? 2 : 4;
  return stride * es % 16 == 0 ? FICOCO_OK : FICOCO_ERR_INVALID_ARG;
}

// The parts of a cache; rows of a call, row offsets and index lists.
Span codes_of(const ficoco_cache* c, const void* codes) { return {codes, (size_t)c->n_pages * c->kv_heads * c->page_size * c->head_dim}; }
Span scales_of(const ficoco_cache* c, const float* scales) { return {scales, (size_t)c->n_pages * c->kv_heads * 4}; }
Span table_of(const ficoco_cache* c) { return {c->page_table, ((size_t)(c->batch - 1) * c->table_stride + c->max_pages) * 4}; }
Span rows_of(const void* p, int rows, long long stride, size_t width, int dtype) {
  return {rows > 0 ? p : nullptr, ((size_t)std::max(rows - 1, 0) * stride + width) * (dtype == FICOCO_BF16 ? 2 : 4)};
}
Span ints_of(const int* p, size_t n) { return {p, n * 4}; }

int check_attention(const ficoco_cache* c, const ficoco_attention_args* a) {
  if (!a || !a->cu_rows || !aligned4(a->cu_rows) || !aligned4(a->lse) || a->heads < 1) return FICOCO_ERR_INVALID_ARG;
  const int rc = check_rows(a->q, a->rows, a->q_stride, a->dtype, (long long)a->heads * c->head_dim);
  if (rc) return rc;
  if (a->heads % c->kv_heads != 0 || a->window < 0 || a->sinks < 0) return FICOCO_ERR_INVALID_ARG;
  if (!(a->scale > 0.f) || !isfinite(a->scale)) return FICOCO_ERR_INVALID_ARG;
  if (a->flags & ~(unsigned)FICOCO_CAUSAL) return FICOCO_ERR_INVALID_ARG;
  if (a->heads > 65535 || (long long)a->rows * a->heads > INT32_MAX) return FICOCO_ERR_UNSUPPORTED;
  return FICOCO_OK;
}
MaskRule mask_rule(const ficoco_attention_args* a) {
  // (a window of 2^30 hides nothing: no sequence is longer)
  return MaskRule{std::min(a->window, 1 << 30), a->window > 0 ? a->sinks : 0, (a->flags & FICOCO_CAUSAL) ? 1 : 0};
}

#define CACHE_TRY(ctx, expr)                                  \
  do {                                                        \
    const cudaError_t e__ = (expr);                           \
    if (e__ != cudaSuccess) return ctx_cuda_error((ctx), e__); \
  } while (0)

// Log2 of the threads of a team that holds `vectors` vectors, `held` each: 32 to half a CTA (two teams at least, a head's keys and
// values).
int team_log(int vectors, int held) {
  int l = 5;
  while (l < PAGE_LOG - 1 && (held << l) < vectors) ++l;
  return l;
}

template <class T, int HELD>
cudaError_t append(const CacheView& c, const ficoco_append_args* a, int rows_held, unsigned* status, cudaStream_t st) {
  const int log_team = team_log(rows_held * c.dim / 8, HELD);
  const dim3 grid(a->rows / c.page + 2 * c.batch, ((2 * c.kv << log_team) + PAGE_THREADS - 1) / PAGE_THREADS);
  return launch(k_cache_append<T, HELD>, grid, PAGE_THREADS, 0, st, c, (const T*)a->k, (const T*)a->v, a->cu_rows, a->k_stride, a->v_stride,
                a->rows, log_team, status);
}

// Tensor maps over the code arrays: rows of head_dim bytes, boxes of a page, the swizzle of a row's width.
typedef CUresult (*encode_fn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                              CUtensorMapFloatOOBfill);
int code_map(ficoco_ctx* ctx, const CacheView& c, const uint8_t* codes, CUtensorMap* map) {
  static const encode_fn encode = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult r;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &r) != cudaSuccess || r != cudaDriverEntryPointSuccess)
      f = nullptr;
    return (encode_fn)f;
  }();
  if (!encode) return ctx_cuda_error(ctx, cudaErrorNotSupported);
  const cuuint64_t dims[2] = {(cuuint64_t)c.dim, (cuuint64_t)c.n_pages * c.kv * c.page}, strides[1] = {(cuuint64_t)c.dim};
  const cuuint32_t box[2] = {(cuuint32_t)c.dim, (cuuint32_t)c.page}, step[2] = {1, 1};
  const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, (void*)codes, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            c.dim == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                            CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? FICOCO_OK : ctx_cuda_error(ctx, cudaErrorInvalidValue);
}

// Scratch for the partial results of cut items: two per CTA, the largest of them.
constexpr int SCRATCH_CTAS_PER_SM = 2;
size_t scratch_bytes(const CtxAccess& x) {
  return (size_t)x.num_sms * SCRATCH_CTAS_PER_SM * 2 * StepPlan<128, 2, 16>::PART * sizeof(float);
}

template <class T, int DIM, int NT, int RB>
int attend_step(ficoco_ctx* ctx, const CtxAccess& x, const CacheView& c, const ficoco_attention_args* a, float scale_log2, int* counters,
                float* partials, cudaStream_t st) {
  using PL = StepPlan<DIM, NT, RB>;
  static_assert(PL::PART <= StepPlan<128, 2, 16>::PART, "the scratch holds it");
  int rc;
  CUtensorMap km, vm;
  if ((rc = code_map(ctx, c, c.k, &km)) || (rc = code_map(ctx, c, c.v, &vm))) return rc;
  CACHE_TRY(ctx, cudaFuncSetAttribute(k_cache_step<T, DIM, NT, RB>, cudaFuncAttributeMaxDynamicSharedMemorySize, PL::SMEM));
  ctx_prof_tick(ctx, st, "k_cache_step");
  CACHE_TRY(ctx, launch(k_cache_step<T, DIM, NT, RB>, dim3(x.num_sms * SCRATCH_CTAS_PER_SM), STEP_THREADS, PL::SMEM, st, km, vm, c,
                        (const T*)a->q, a->cu_rows, (T*)a->out, a->lse, a->q_stride, scale_log2, a->rows, a->heads, mask_rule(a),
                        counters, partials, x.status, x.wait_ns, x.extra_arrivals));
  ctx_prof_tick(ctx, st, nullptr);
  ctx_set_launches(ctx, 1);
  return FICOCO_OK;
}
template <int DIM>
int attend_prompt(ficoco_ctx* ctx, const CtxAccess& x, const CacheView& c, const ficoco_attention_args* a, float scale_log2, cudaStream_t st) {
  using PL = PromptPlan<DIM>;
  CUtensorMap km, vm;
  int rc;
  if ((rc = code_map(ctx, c, c.k, &km)) || (rc = code_map(ctx, c, c.v, &vm))) return rc;
  CACHE_TRY(ctx, cudaFuncSetAttribute(k_cache_prompt<DIM>, cudaFuncAttributeMaxDynamicSharedMemorySize, PL::SMEM));
  const long long units = (long long)a->rows * (a->heads / c.kv) / PROMPT_ROWS + c.batch;
  ctx_prof_tick(ctx, st, "k_cache_prompt");
  CACHE_TRY(ctx, launch(k_cache_prompt<DIM>, dim3((unsigned)(units * c.kv)), PROMPT_THREADS, PL::SMEM, st, km, vm, c,
                        (const __nv_bfloat16*)a->q, a->cu_rows, (__nv_bfloat16*)a->out, a->lse, a->q_stride, scale_log2, a->rows, a->heads,
                        mask_rule(a), x.status, x.wait_ns, x.extra_arrivals));
  ctx_prof_tick(ctx, st, nullptr);
  ctx_set_launches(ctx, 1);
  return FICOCO_OK;
}
template <int DIM>
int attend_dim(ficoco_ctx* ctx, const CtxAccess& x, const CacheView& c, const ficoco_attention_args* a, float scale_log2, bool listed,
               cudaStream_t st) {
  int* counters;
  float* partials;
  // (also where a prompt needs none: so the first call, whatever its rows, is the one that allocates)
  const int rc = ctx_cache_scratch(ctx, st, scratch_bytes(x), &counters, &partials);
  if (rc) return rc;
  if (a->dtype == FICOCO_FP32) return attend_step<float, DIM, 6, 8>(ctx, x, c, a, scale_log2, counters, partials, st);
  const long long rows = (long long)a->rows * (a->heads / c.kv);       // of all sequences, per key/value head
  // The prompt kernel takes 256 rows per CTA and needs about 5000 cycles for a tile of tokens, one CTA per SM; the step kernel takes 16
  // rows per item, two CTAs per SM, about 3000 cycles a tile: whichever has the shorter line (the tiles per row are the same).  Sequences that
  // open a CTA for less than 256 rows are not counted one by one: their tiles hold 128 rows at most and take less (prompt / step kernel, us: 128
  // sequences of 40 rows, 640 tokens, 32 heads 558 / 767, with 8 key/value heads 185 / 646; 600 of 12 rows, 32 heads on 8, 593 / 783).
  const long long prompt_ctas = std::max(1ll, rows / PROMPT_ROWS) * c.kv, step_items = (rows / 16 + 1) * c.kv;
  const long long prompt_time = (prompt_ctas + x.num_sms - 1) / x.num_sms * 5000, step_time = step_items * 3000 / (2 * x.num_sms);
  if (!listed || (rows > 32ll * c.batch && prompt_time < step_time)) return attend_prompt<DIM>(ctx, x, c, a, scale_log2, st);
  if (rows <= 8ll * c.batch) return attend_step<__nv_bfloat16, DIM, 2, 8>(ctx, x, c, a, scale_log2, counters, partials, st);
  return attend_step<__nv_bfloat16, DIM, 2, 16>(ctx, x, c, a, scale_log2, counters, partials, st);
}

template <class T, int DIM, int NT, int RC>
int weigh(ficoco_ctx* ctx, const CtxAccess& x, const CacheView& c, const ficoco_attention_args* a, int n_text, int first, int count,
          float* weights, float scale_log2, cudaStream_t st) {
  using PL = WeightPlan<DIM, NT, RC>;
  CUtensorMap km;
  const int rc = code_map(ctx, c, c.k, &km);
  if (rc) return rc;
  CACHE_TRY(ctx, cudaFuncSetAttribute(k_cache_weights<T, DIM, NT, RC>, cudaFuncAttributeMaxDynamicSharedMemorySize, PL::SMEM));
  const int chunks = (int)(((long long)n_text * (a->heads / c.kv) + RC - 1) / RC);
  const int tiles = (int)(((long long)first + count + CTILE - 1) / CTILE - first / CTILE);
  const long long total = (long long)chunks * c.batch * c.kv * tiles;
  ctx_prof_tick(ctx, st, "k_cache_weights");
  CACHE_TRY(ctx, launch(k_cache_weights<T, DIM, NT, RC>, dim3((unsigned)std::min<long long>(total, 2ll * x.num_sms)), WEIGHT_THREADS, PL::SMEM, st,
                        km, c, (const T*)a->q, a->cu_rows, a->lse, weights, a->q_stride, scale_log2, a->rows, a->heads, mask_rule(a),
                        n_text, first, count, tiles, chunks, x.status, x.wait_ns, x.extra_arrivals));
  ctx_prof_tick(ctx, st, nullptr);
  ctx_set_launches(ctx, 1);
  return FICOCO_OK;
}
template <int DIM>
int weigh_dim(ficoco_ctx* ctx, const CtxAccess& x, const CacheView& c, const ficoco_attention_args* a, int n_text, int first, int count,
              float* weights, float scale_log2, cudaStream_t st) {
  if (a->dtype == FICOCO_FP32) return weigh<float, DIM, 6, 16>(ctx, x, c, a, n_text, first, count, weights, scale_log2, st);
  return weigh<__nv_bfloat16, DIM, 2, 64>(ctx, x, c, a, n_text, first, count, weights, scale_log2, st);
}

}  // namespace

extern "C" int ficoco_cache_append(ficoco_ctx* ctx, const ficoco_cache* cache, const ficoco_append_args* a, void* cuda_stream) {
  if (!ctx || !a) return FICOCO_ERR_INVALID_ARG;
  CacheView c;
  int rc = check_cache(cache, &c);
  if (rc) return rc;
  if (!a->cu_rows || !aligned4(a->cu_rows)) return FICOCO_ERR_INVALID_ARG;
  const long long width = (long long)c.kv * c.dim;
  if ((rc = check_rows(a->k, a->rows, a->k_stride, a->dtype, width)) || (rc = check_rows(a->v, a->rows, a->v_stride, a->dtype, width))) return rc;
  if (overlap({codes_of(cache, cache->k_codes), codes_of(cache, cache->v_codes), scales_of(cache, cache->k_scale), scales_of(cache, cache->v_scale)},
              {rows_of(a->k, a->rows, a->k_stride, width, a->dtype), rows_of(a->v, a->rows, a->v_stride, width, a->dtype), table_of(cache),
               ints_of(cache->lengths, c.batch), ints_of(a->cu_rows, c.batch + 1)}))
    return FICOCO_ERR_INVALID_ARG;
  const CtxAccess x = ctx_access(ctx);
  cudaStream_t st = (cudaStream_t)cuda_stream;
  CACHE_TRY(ctx, cudaSetDevice(x.device));
  ctx_set_launches(ctx, 0);
  if (a->rows == 0) return FICOCO_OK;
  ctx_prof_tick(ctx, st, "k_cache_append");
  // teams that hold a full page, or, where few rows come per sequence, four rows (longer ones are read twice)
  const bool few = a->rows <= 4ll * c.batch, bf16 = a->dtype == FICOCO_BF16;
  CACHE_TRY(ctx, few ? (bf16 ? append<__nv_bfloat16, STEP_HELD>(c, a, 4, x.status, st) : append<float, STEP_HELD>(c, a, 4, x.status, st))
                     : (bf16 ? append<__nv_bfloat16, APPEND_HELD>(c, a, c.page, x.status, st)
                             : append<float, APPEND_HELD>(c, a, c.page, x.status, st)));
  ctx_prof_tick(ctx, st, nullptr);
  ctx_set_launches(ctx, 1);
  return FICOCO_OK;
}

extern "C" int ficoco_cache_attention(ficoco_ctx* ctx, const ficoco_cache* cache, const ficoco_attention_args* a, void* cuda_stream) {
  if (!ctx) return FICOCO_ERR_INVALID_ARG;
  CacheView c;
  int rc = check_cache(cache, &c);
  if (rc || (rc = check_attention(cache, a))) return rc;
  if ((a->rows > 0 && !a->out) || !aligned16(a->out)) return FICOCO_ERR_INVALID_ARG;
  const size_t width = (size_t)a->heads * c.dim;
  const Span q = rows_of(a->q, a->rows, a->q_stride, width, a->dtype), out = rows_of(a->out, a->rows, width, width, a->dtype);
  const Span lse = {a->rows > 0 ? a->lse : nullptr, (size_t)a->rows * a->heads * 4};
  if (overlap({out, lse}, {q, codes_of(cache, cache->k_codes), codes_of(cache, cache->v_codes), scales_of(cache, cache->k_scale),
                           scales_of(cache, cache->v_scale), table_of(cache), ints_of(cache->lengths, c.batch), ints_of(a->cu_rows, c.batch + 1)}) ||
      overlap(out, lse))
    return FICOCO_ERR_INVALID_ARG;
  const CtxAccess x = ctx_access(ctx);
  cudaStream_t st = (cudaStream_t)cuda_stream;
  CACHE_TRY(ctx, cudaSetDevice(x.device));
  ctx_set_launches(ctx, 0);
  if (a->rows == 0) return FICOCO_OK;
  const float scale_log2 = a->scale * 1.4426950408889634f;
  // The step kernel's list of tiles, of 8 rows by 128 tokens, is counted in 32 bits.  What its table's room could make longer takes the kernel
  // of prompts, which has no list, or, with few rows or fp32, the kernel without tiles (one sequence of 4096 tokens, 32 heads on 8, 64 rows:
  // 84 us, without tiles 836; 2944 rows: 175 and 22900).
  const double most_tiles = ((double)a->rows * (a->heads / c.kv) / 8 + c.batch) * c.kv * ((double)c.max_pages * c.page / CTILE + 2);
  const bool listed = most_tiles < 2e9;
  if (listed || (a->dtype == FICOCO_BF16 && (long long)a->rows * (a->heads / c.kv) > 32ll * c.batch)) {
    if (c.dim == 128) return attend_dim<128>(ctx, x, c, a, scale_log2, listed, st);
    if (c.dim == 64) return attend_dim<64>(ctx, x, c, a, scale_log2, listed, st);
  }
  const dim3 grid(a->rows, a->heads);
  ctx_prof_tick(ctx, st, "k_cache_attention_simt");
  if (a->dtype == FICOCO_BF16)
    CACHE_TRY(ctx, launch(k_cache_attention_simt<__nv_bfloat16>, grid, CS_THREADS, 0, st, c, (const __nv_bfloat16*)a->q,
                          a->cu_rows, (__nv_bfloat16*)a->out, a->lse, a->q_stride, scale_log2, a->rows, a->heads,
                          mask_rule(a), x.status));
  else
    CACHE_TRY(ctx, launch(k_cache_attention_simt<float>, grid, CS_THREADS, 0, st, c, (const float*)a->q, a->cu_rows,
                          (float*)a->out, a->lse, a->q_stride, scale_log2, a->rows, a->heads, mask_rule(a), x.status));
  ctx_prof_tick(ctx, st, nullptr);
  ctx_set_launches(ctx, 1);
  return FICOCO_OK;
}

extern "C" int ficoco_cache_weights(ficoco_ctx* ctx, const ficoco_cache* cache, const ficoco_attention_args* a, int n_text,
                                    int first, int count, float* weights, void* cuda_stream) {
  if (!ctx) return FICOCO_ERR_INVALID_ARG;
  CacheView c;
  int rc = check_cache(cache, &c);
  if (rc || (rc = check_attention(cache, a))) return rc;
  if ((a->rows > 0 && !a->lse) || !weights || !aligned4(weights) || n_text < 1 || first < 0 || count < 1) return FICOCO_ERR_INVALID_ARG;
  if ((long long)c.batch * n_text > INT32_MAX || (long long)first + count > INT32_MAX) return FICOCO_ERR_UNSUPPORTED;
  const double bytes = 4.0 * c.batch * a->heads * n_text * count;
  if (overlap({Span{weights, (size_t)std::min(bytes, 1e18)}},
              {rows_of(a->q, a->rows, a->q_stride, (size_t)a->heads * c.dim, a->dtype), Span{a->rows > 0 ? a->lse : nullptr, (size_t)a->rows * a->heads * 4},
               codes_of(cache, cache->k_codes), scales_of(cache, cache->k_scale), table_of(cache), ints_of(cache->lengths, c.batch),
               ints_of(a->cu_rows, c.batch + 1)}))
    return FICOCO_ERR_INVALID_ARG;
  const CtxAccess x = ctx_access(ctx);
  cudaStream_t st = (cudaStream_t)cuda_stream;
  CACHE_TRY(ctx, cudaSetDevice(x.device));
  const float scale_log2 = a->scale * 1.4426950408889634f;
  // (items are counted and a head group's weights are indexed in 32 bits; what exceeds either takes the kernel without tiles)
  if ((double)c.batch * c.kv * ((double)n_text * (a->heads / c.kv) / 16 + 1) < 2e9 &&
      (double)n_text * (a->heads / c.kv) * count + first + count < 4e9 &&
      ((double)n_text * (a->heads / c.kv) + 64) * n_text < 4e9) {
    if (c.dim == 128) return weigh_dim<128>(ctx, x, c, a, n_text, first, count, weights, scale_log2, st);
    if (c.dim == 64) return weigh_dim<64>(ctx, x, c, a, n_text, first, count, weights, scale_log2, st);
  }
  const dim3 grid(c.batch * n_text, a->heads);
  ctx_prof_tick(ctx, st, "k_cache_weights_simt");
  if (a->dtype == FICOCO_BF16)
    CACHE_TRY(ctx, launch(k_cache_weights_simt<__nv_bfloat16>, grid, CS_THREADS, 0, st, c, (const __nv_bfloat16*)a->q,
                          a->cu_rows, a->lse, weights, a->q_stride, scale_log2, a->rows, a->heads, mask_rule(a), n_text,
                          first, count, x.status));
  else
    CACHE_TRY(ctx, launch(k_cache_weights_simt<float>, grid, CS_THREADS, 0, st, c, (const float*)a->q, a->cu_rows, a->lse,
                          weights, a->q_stride, scale_log2, a->rows, a->heads, mask_rule(a), n_text, first, count, x.status));
  ctx_prof_tick(ctx, st, nullptr);
  ctx_set_launches(ctx, 1);
  return FICOCO_OK;
}

extern "C" int ficoco_cache_copy(ficoco_ctx* ctx, const ficoco_cache* cache, const int* src, const int* dst, int n, void* cuda_stream) {
  if (!ctx) return FICOCO_ERR_INVALID_ARG;
  CacheView c;
  const int rc = check_cache(cache, &c);
  if (rc) return rc;
  if (n < 0 || (n > 0 && (!src || !dst || src == dst || !aligned4(src) || !aligned4(dst)))) return FICOCO_ERR_INVALID_ARG;
  if (n > 0 && overlap({codes_of(cache, cache->k_codes), codes_of(cache, cache->v_codes), scales_of(cache, cache->k_scale),
                        scales_of(cache, cache->v_scale)}, {ints_of(src, n), ints_of(dst, n)}))
    return FICOCO_ERR_INVALID_ARG;
  const CtxAccess x = ctx_access(ctx);
  cudaStream_t st = (cudaStream_t)cuda_stream;
  CACHE_TRY(ctx, cudaSetDevice(x.device));
  ctx_set_launches(ctx, 0);
  if (n == 0) return FICOCO_OK;
  const size_t words = (size_t)c.kv * c.page * c.dim / 16;        // at most 2 M (1024 heads x 128 tokens x 256)
  const int parts = (int)std::min<size_t>(std::max<size_t>(1, words / (4 * COPY_THREADS)), 64);
  ctx_prof_tick(ctx, st, "k_cache_copy");
  CACHE_TRY(ctx, launch(k_cache_copy, dim3(n, parts), COPY_THREADS, 0, st, c, src, dst, (int)words, x.status));
  ctx_prof_tick(ctx, st, nullptr);
  ctx_set_launches(ctx, 1);
  return FICOCO_OK;
}

extern "C" int ficoco_cache_compact(ficoco_ctx* ctx, const ficoco_cache* cache, const ficoco_compact_args* a, void* cuda_stream) {
  if (!ctx || !a) return FICOCO_ERR_INVALID_ARG;
  CacheView c;
  const int rc = check_cache(cache, &c);
  if (rc) return rc;
  if (!a->to_table || !a->cu_kept || a->n_kept < 0 || (a->n_kept > 0 && !a->kept) || a->first < 0 || a->to_pages < 1 ||
      a->to_stride < a->to_pages || a->to_table == c.table || a->lengths_out == c.len)
    return FICOCO_ERR_INVALID_ARG;
  if (!aligned4(a->to_table) || !aligned4(a->kept) || !aligned4(a->cu_kept) || !aligned4(a->lengths_out)) return FICOCO_ERR_INVALID_ARG;
  if ((long long)a->n_kept + (long long)c.batch * a->first > INT32_MAX / 2) return FICOCO_ERR_UNSUPPORTED;
  const Span lengths_out = ints_of(a->lengths_out, c.batch);
  if (overlap({codes_of(cache, cache->k_codes), codes_of(cache, cache->v_codes), scales_of(cache, cache->k_scale), scales_of(cache, cache->v_scale),
               lengths_out},
              {Span{a->to_table, ((size_t)(c.batch - 1) * a->to_stride + a->to_pages) * 4}, ints_of(a->n_kept > 0 ? a->kept : nullptr, a->n_kept),
               ints_of(a->cu_kept, c.batch + 1), table_of(cache), ints_of(cache->lengths, c.batch)}) ||
      overlap({lengths_out}, {codes_of(cache, cache->k_codes), codes_of(cache, cache->v_codes), scales_of(cache, cache->k_scale),
                              scales_of(cache, cache->v_scale)}))
    return FICOCO_ERR_INVALID_ARG;
  const CtxAccess x = ctx_access(ctx);
  cudaStream_t st = (cudaStream_t)cuda_stream;
  CACHE_TRY(ctx, cudaSetDevice(x.device));
  const int log_team = team_log(c.page * c.dim / 16, COMPACT_HELD);
  const long long units = ((long long)a->n_kept + (long long)c.batch * a->first) / c.page + 2 * c.batch;
  // CTAs along the heads of a page: as few as leave every SM eight (48 gathered sequences of 32 heads in pages of 16: 153 us, with one
  // CTA per head group 208; 16 sequences in pages of 64 14.6, with one per head group 16.5)
  const int parts = ((2 * c.kv << log_team) + PAGE_THREADS - 1) / PAGE_THREADS;
  const dim3 grid((unsigned)units, (unsigned)std::min<long long>(parts, std::max(1ll, (8ll * x.num_sms + units - 1) / units)));
  ctx_prof_tick(ctx, st, "k_cache_compact");
  CACHE_TRY(ctx, launch(k_cache_compact, grid, PAGE_THREADS, 0, st, c, a->to_table, a->kept, a->cu_kept, a->lengths_out,
                        a->to_stride, a->to_pages, a->n_kept, a->first, log_team, x.status));
  ctx_prof_tick(ctx, st, nullptr);
  ctx_set_launches(ctx, 1);
  return FICOCO_OK;
}

// ---- page pool (host) ---------------------------------------------------------------------------------------------
struct ficoco_pool {
  std::vector<int> holders;                                                     // per page; 0: free
  std::priority_queue<int, std::vector<int>, std::greater<int>> free_pages;     // lowest first
};

extern "C" int ficoco_pool_create(ficoco_pool** out, int n_pages) {
  if (!out || n_pages < 1) return FICOCO_ERR_INVALID_ARG;
  try {
    ficoco_pool* p = new ficoco_pool();
    try {
      p->holders.assign(n_pages, 0);
      std::vector<int> all(n_pages);
      for (int i = 0; i < n_pages; ++i) all[i] = i;
      p->free_pages = decltype(p->free_pages)(std::greater<int>(), std::move(all));
    } catch (...) {
      delete p;
      throw;
    }
    *out = p;
    return FICOCO_OK;
  } catch (...) {                                     // out of memory: nothing crosses the C boundary
    return FICOCO_ERR_PAGES;
  }
}

extern "C" int ficoco_pool_destroy(ficoco_pool* p) {
  if (!p) return FICOCO_ERR_INVALID_ARG;
  delete p;
  return FICOCO_OK;
}

extern "C" int ficoco_pool_free_pages(const ficoco_pool* p) { return p ? (int)p->free_pages.size() : FICOCO_ERR_INVALID_ARG; }

extern "C" int ficoco_pool_take(ficoco_pool* p, int n, int* pages) {
  if (!p || n < 0 || (n > 0 && !pages)) return FICOCO_ERR_INVALID_ARG;
  if ((size_t)n > p->free_pages.size()) return FICOCO_ERR_PAGES;
  for (int i = 0; i < n; ++i) {
    pages[i] = p->free_pages.top();
    p->free_pages.pop();
    p->holders[pages[i]] = 1;
  }
  return FICOCO_OK;
}

extern "C" int ficoco_pool_give(ficoco_pool* p, int n, const int* pages) {
  if (!p || n < 0 || (n > 0 && !pages)) return FICOCO_ERR_INVALID_ARG;
  // all or nothing: a list may hold a page as often as it has holders
  int done = 0;
  for (; done < n; ++done) {
    const int g = pages[done];
    if (g < 0 || g >= (int)p->holders.size() || p->holders[g] < 1) break;
    --p->holders[g];
  }
  if (done < n) {
    while (done-- > 0) ++p->holders[pages[done]];
    return FICOCO_ERR_PAGES;
  }
  try {
    for (int i = 0; i < n; ++i) {
      const int g = pages[i];
      if (p->holders[g] != 0) continue;
      p->holders[g] = -1;                             // (so that a page given twice in one list is queued once)
      p->free_pages.push(g);
    }
  } catch (...) {
  }
  for (int i = 0; i < n; ++i)
    if (p->holders[pages[i]] < 0) p->holders[pages[i]] = 0;
  return FICOCO_OK;
}

extern "C" int ficoco_pool_fork(ficoco_pool* p, int page_size, int length, const int* pages, int* forked, int* copy_from,
                                int* copy_to) {
  if (!p || page_size < 1 || length < 0 || !copy_from || !copy_to) return FICOCO_ERR_INVALID_ARG;
  *copy_from = *copy_to = -1;
  const int full = length / page_size, part = length % page_size ? 1 : 0;
  if (full + part == 0) return FICOCO_OK;
  if (!pages || !forked) return FICOCO_ERR_INVALID_ARG;
  for (int i = 0; i < full + part; ++i)
    if (pages[i] < 0 || pages[i] >= (int)p->holders.size() || p->holders[pages[i]] < 1) return FICOCO_ERR_PAGES;
  if (part && p->free_pages.empty()) return FICOCO_ERR_PAGES;
  for (int i = 0; i < full; ++i) {
    forked[i] = pages[i];
    ++p->holders[pages[i]];
  }
  if (part) {
    const int rc = ficoco_pool_take(p, 1, copy_to);
    if (rc) return rc;
    *copy_from = pages[full];
    forked[full] = *copy_to;
  }
  return FICOCO_OK;
}
