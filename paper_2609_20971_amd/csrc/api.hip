// C ABI of librbs: argument validation, then kernel launches on the caller's
// stream.  Validation is host-only and happens before any HIP call, so a
// rejected call launches and writes nothing.
#include <math.h>
#include <stdint.h>
#include <stdlib.h>
#include <string.h>

#include <atomic>

#include "../../include/rbs.h"
#include "paged.hpp"
#include "rbs_launch.hpp"

namespace {

constexpr int kMaxTokens = 262144;
constexpr int kMaxHeads = 512;  // query heads of the calls around the paged cache

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int blocks_of(const rbs_shape* s) { return (s->n_tokens + s->block_size - 1) / s->block_size; }

constexpr int64_t kMaxTokStride = int64_t(1) << 23;  // (B - 1) rows of it, in bytes, fit the copies' 32-bit offsets

// Strides of one tensor of H heads and T tokens of d = 128 (zero: the dense
// value), validated: multiples of 8 elements (16-byte rows), token strides
// within kMaxTokStride, and rows of distinct (head, token) pairs disjoint
// (head-major or token-major nesting).
int resolve_strides(int64_t head_in, int64_t tok_in, int H, int64_t T, int64_t* head, int64_t* tok) {
  const int64_t st = tok_in == 0 ? 128 : tok_in;
  const int64_t sh = head_in == 0 ? T * 128 : head_in;
  if (st < 0 || sh < 0 || st % 8 != 0 || sh % 8 != 0 || st > kMaxTokStride) return RBS_ERR_SHAPE;
  const bool head_major = st >= 128 && sh >= T * st;
  const bool tok_major = sh >= 128 && st >= (int64_t)H * sh;
  if (!head_major && !tok_major) return RBS_ERR_SHAPE;
  *head = sh;
  *tok = st;
  return RBS_OK;
}

// The strides of Q (and O) and of K and V, resolved and validated.
int strides_of(const rbs_shape* s, rbs::Strides* out) {
  int rc = resolve_strides(s->q_stride_head, s->q_stride_tok, s->n_q_heads, s->n_tokens, &out->q_head, &out->q_tok);
  if (rc != RBS_OK) return rc;
  return resolve_strides(s->kv_stride_head, s->kv_stride_tok, s->n_kv_heads, s->n_tokens, &out->kv_head,
                         &out->kv_tok);
}

int check_shape(const rbs_shape* s) {
  if (s == nullptr) return RBS_ERR_NULL;
  if (s->head_dim != 128) return RBS_ERR_UNSUPPORTED;
  if (s->block_size != 64 && s->block_size != 128 && s->block_size != 256) return RBS_ERR_UNSUPPORTED;
  if (s->n_tokens < 1 || s->n_tokens > kMaxTokens) return RBS_ERR_SHAPE;
  if (s->n_q_heads < 1 || s->n_kv_heads < 1) return RBS_ERR_SHAPE;
  if (s->n_q_heads % s->n_kv_heads != 0) return RBS_ERR_SHAPE;
  if (blocks_of(s) > rbs::kMaxBlocks) return RBS_ERR_SHAPE;
  if ((int64_t)s->n_q_heads * blocks_of(s) > INT32_MAX / 2) return RBS_ERR_SHAPE;
  rbs::Strides st;
  return strides_of(s, &st);
}

int check_stats_ptrs(const rbs_stats* st) {
  if (st == nullptr || st->centroids == nullptr || st->radii == nullptr || st->beta == nullptr ||
      st->quantiles == nullptr || st->summary == nullptr)
    return RBS_ERR_NULL;
  if (!aligned16(st->centroids) || !aligned16(st->radii) || !aligned16(st->beta) || !aligned16(st->quantiles) ||
      !aligned16(st->summary))
    return RBS_ERR_ALIGN;
  return RBS_OK;
}

int from_hip(hipError_t e) { return e == hipSuccess ? RBS_OK : RBS_ERR_HIP; }

// ---- Debug mode: synchronise after every call, and scan Q before selection.
std::atomic<int> g_debug{-1};  // -1: the environment not read yet

bool debug_on() {
  int d = g_debug.load(std::memory_order_relaxed);
  if (d < 0) {
    const char* e = getenv("RBS_DEBUG");
    int fresh = (e != nullptr && e[0] != '\0' && strcmp(e, "0") != 0) ? 1 : 0;
    int expected = -1;
    g_debug.compare_exchange_strong(expected, fresh);
    d = g_debug.load(std::memory_order_relaxed);
  }
  return d > 0;
}

// The status of a call whose launches returned e: in debug mode the stream is
// drained and any kernel failure reported.
int finish(hipError_t e, void* stream) {
  if (e != hipSuccess) return RBS_ERR_HIP;
  if (!debug_on()) return RBS_OK;
  if (hipStreamSynchronize(static_cast<hipStream_t>(stream)) != hipSuccess) return RBS_ERR_HIP;
  return hipGetLastError() == hipSuccess ? RBS_OK : RBS_ERR_HIP;
}

__device__ unsigned int g_q_range_flag;

// One thread per 16-byte chunk of Q ([H][N][128] through the strides): sets
// the flag if a bf16 element's magnitude is 65536 or more (bits & 0x7fff >=
// 0x4780: beyond f16's 65504, infinities and NaNs included).
__global__ __launch_bounds__(256) void q_range_kernel(const uint16_t* __restrict__ Q, int64_t head, int64_t tok,
                                                      int N, int64_t chunks) {
  const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (c >= chunks) return;
  const int64_t row = c >> 4;
  const int64_t h = row / N, t = row - h * N;
  const uint4 v = *reinterpret_cast<const uint4*>(Q + h * head + t * tok + 8 * (c & 15));
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  bool bad = false;
#pragma unroll
  for (int k = 0; k < 4; ++k) bad |= (w[k] & 0x7fffu) >= 0x4780u || ((w[k] >> 16) & 0x7fffu) >= 0x4780u;
  if (bad) atomicOr(&g_q_range_flag, 1u);
}

// Debug mode only: RBS_ERR_RANGE if Q holds an element the selector's f16
// operands cannot represent.
int check_q_range(const void* Q, int64_t head, int64_t tok, int H, int N, void* stream) {
  if (!debug_on()) return RBS_OK;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const unsigned int zero = 0u;
  if (hipStreamSynchronize(s) != hipSuccess) return RBS_ERR_HIP;
  if (hipMemcpyToSymbol(HIP_SYMBOL(g_q_range_flag), &zero, sizeof zero) != hipSuccess) return RBS_ERR_HIP;
  const int64_t chunks = (int64_t)H * N * 16;
  hipLaunchKernelGGL(q_range_kernel, dim3((unsigned)((chunks + 255) / 256)), dim3(256), 0, s,
                     static_cast<const uint16_t*>(Q), head, tok, N, chunks);
  if (hipGetLastError() != hipSuccess || hipStreamSynchronize(s) != hipSuccess) return RBS_ERR_HIP;
  unsigned int flag = 0u;
  if (hipMemcpyFromSymbol(&flag, HIP_SYMBOL(g_q_range_flag), sizeof flag) != hipSuccess) return RBS_ERR_HIP;
  return flag != 0u ? RBS_ERR_RANGE : RBS_OK;
}

// Shape rules of a batch (the per-sequence limits are the single-sequence
// ones), and its sequence table.  T = shape->n_tokens must equal the sum.
int check_batch(const rbs_shape* s, const rbs_batch* b, rbs::SeqTable* t) {
  if (s == nullptr || b == nullptr || b->seq_tokens == nullptr) return RBS_ERR_NULL;
  if (s->head_dim != 128) return RBS_ERR_UNSUPPORTED;
  if (s->block_size != 64 && s->block_size != 128 && s->block_size != 256) return RBS_ERR_UNSUPPORTED;
  if (s->n_q_heads < 1 || s->n_kv_heads < 1 || s->n_q_heads % s->n_kv_heads != 0) return RBS_ERR_SHAPE;
  if (b->n_seqs < 1 || b->n_seqs > RBS_MAX_SEQS) return RBS_ERR_SHAPE;
  static_assert(RBS_MAX_SEQS == rbs::kMaxSeqs, "sequence table size");
  static_assert(RBS_ATTN_WORKSPACE_BYTES == rbs::kQueueInts * sizeof(int), "attention workspace size");
  *t = rbs::SeqTable{};
  t->n = b->n_seqs;
  int64_t tok = 0, blk = 0, cap = 0;
  for (int q = 0; q < b->n_seqs; ++q) {
    const int64_t n = b->seq_tokens[q];
    if (n < 1 || n > kMaxTokens) return RBS_ERR_SHAPE;
    const int64_t m = (n + s->block_size - 1) / s->block_size;
    if (m > rbs::kMaxBlocks) return RBS_ERR_SHAPE;
    tok += n;
    blk += m;
    cap += m * (m + 1) / 2;
    t->tok[q + 1] = (int)tok;
    t->blk[q + 1] = (int)blk;
    t->cap[q + 1] = cap;
  }
  if (tok != s->n_tokens) return RBS_ERR_SHAPE;
  if ((int64_t)s->n_q_heads * blk > INT32_MAX / 2) return RBS_ERR_SHAPE;
  rbs::Strides st;
  return strides_of(s, &st);
}

// ---- Paged cache.

// log2 of a page size, or -1 if it is not one of 16 .. 256.
int page_shift_of(int32_t page_size) {
  for (int s = 4; s <= 8; ++s)
    if (page_size == 1 << s) return s;
  return -1;
}

int check_cache(const rbs_cache* c, rbs::CacheView* out) {
  if (c == nullptr) return RBS_ERR_NULL;
  const int shift = page_shift_of(c->page_size);
  if (c->head_dim != 128 || shift < 0) return RBS_ERR_UNSUPPORTED;
  if (c->format != RBS_CACHE_BF16 && c->format != RBS_CACHE_FP8) return RBS_ERR_ARG;
  if (c->n_kv_heads < 1 || c->n_pages < 1 || c->n_pages > (INT32_MAX >> shift)) return RBS_ERR_SHAPE;
  rbs::CacheView v{};
  v.tok = c->stride_tok == 0 ? 128 : c->stride_tok;
  v.head = c->stride_head == 0 ? (int64_t)c->page_size * 128 : c->stride_head;
  v.page = c->stride_page == 0 ? (int64_t)c->n_kv_heads * c->page_size * 128 : c->stride_page;
  if (v.tok < 128 || v.head < 128 || v.page < 128 || v.tok % 16 != 0 || v.head % 16 != 0 || v.page % 16 != 0)
    return RBS_ERR_SHAPE;
  // The largest offset (in bytes) has to fit 63 bits, and a place's inside its page the kernels' 31.
  if (v.tok > INT32_MAX / 1024 || v.head > (int64_t(1) << 40) || v.page > (int64_t(1) << 60) / c->n_pages)
    return RBS_ERR_SHAPE;
  if (c->K == nullptr || c->V == nullptr || (c->format == RBS_CACHE_FP8 && c->amax == nullptr)) return RBS_ERR_NULL;
  if (!aligned16(c->K) || !aligned16(c->V) || (c->format == RBS_CACHE_FP8 && !aligned16(c->amax)))
    return RBS_ERR_ALIGN;
  v.K = c->K;
  v.V = c->V;
  v.amax = c->format == RBS_CACHE_FP8 ? c->amax : nullptr;
  v.n_pages = c->n_pages;
  v.page_shift = shift;
  *out = v;
  return RBS_OK;
}

int check_pages(const rbs_pages* p, int* shift) {
  if (p == nullptr) return RBS_ERR_NULL;
  *shift = page_shift_of(p->page_size);
  if (*shift < 0) return RBS_ERR_UNSUPPORTED;
  if (p->n_rows < 1 || p->n_rows > RBS_MAX_ROWS || p->max_pages < 1 || p->max_pages > (INT32_MAX >> *shift) ||
      p->n_pages < 1 || p->n_pages > (INT32_MAX >> *shift))
    return RBS_ERR_SHAPE;
  if (p->page_table == nullptr || p->free_pages == nullptr) return RBS_ERR_NULL;
  if (!aligned16(p->page_table) || !aligned16(p->free_pages)) return RBS_ERR_ALIGN;
  return RBS_OK;
}

// Sizes and strides of the calls around the cache: as check_shape, without its
// rules on blocks and with its own limit on tokens.
int check_heads(const rbs_shape* s, int max_tokens) {
  if (s == nullptr) return RBS_ERR_NULL;
  if (s->head_dim != 128) return RBS_ERR_UNSUPPORTED;
  if (s->n_tokens < 1 || s->n_tokens > max_tokens || s->n_q_heads < 1 || s->n_kv_heads < 1 ||
      s->n_q_heads > kMaxHeads || s->n_q_heads % s->n_kv_heads != 0)
    return RBS_ERR_SHAPE;
  return RBS_OK;
}

// Byte offset of the half-widths in the box summary (centres first, 256-aligned).
size_t box_half_offset(int n_kv_heads, int n_blocks) {
  return ((size_t)n_kv_heads * n_blocks * 128 * sizeof(_Float16) + 255) & ~(size_t)255;
}

}  // namespace

extern "C" {

size_t rbs_summary_bytes(const rbs_shape* shape) {
  if (check_shape(shape) != RBS_OK) return 0;
  return rbs::summary_bytes(shape->n_kv_heads, blocks_of(shape));
}

int64_t rbs_index_capacity(int32_t n_blocks) {
  if (n_blocks < 0) return 0;
  return (int64_t)n_blocks * (n_blocks + 1) / 2;
}

size_t rbs_attention_workspace_bytes(void) { return RBS_ATTN_WORKSPACE_BYTES; }

int rbs_block_stats(const rbs_shape* shape, const void* K, const rbs_stats* stats, void* stream) {
  int rc = check_shape(shape);
  if (rc != RBS_OK) return rc;
  if (K == nullptr) return RBS_ERR_NULL;
  if ((rc = check_stats_ptrs(stats)) != RBS_OK) return rc;
  if (!aligned16(K)) return RBS_ERR_ALIGN;
  const int M = blocks_of(shape);
  rbs::Strides st;
  strides_of(shape, &st);
  rbs::StatsArgs a;
  a.K = static_cast<const uint16_t*>(K);
  a.kv_head = st.kv_head;
  a.kv_tok = st.kv_tok;
  a.n_tokens = shape->n_tokens;
  a.n_kv_heads = shape->n_kv_heads;
  a.block_size = shape->block_size;
  a.n_blocks = M;
  a.centroids = stats->centroids;
  a.radii = stats->radii;
  a.beta = stats->beta;
  a.quantiles = stats->quantiles;
  a.cent16 = static_cast<_Float16*>(stats->summary);
  a.uplift = reinterpret_cast<float*>(static_cast<unsigned char*>(stats->summary) +
                                      rbs::summary_uplift_offset(shape->n_kv_heads, M));
  a.cnorm = reinterpret_cast<float*>(static_cast<unsigned char*>(stats->summary) +
                                     rbs::summary_cnorm_offset(shape->n_kv_heads, M));
  return finish(rbs::launch_stats(a, static_cast<hipStream_t>(stream)), stream);
}

int rbs_stats_summarize(const rbs_shape* shape, const rbs_stats* stats, void* stream) {
  int rc = check_shape(shape);
  if (rc != RBS_OK) return rc;
  if (stats == nullptr || stats->centroids == nullptr || stats->radii == nullptr || stats->beta == nullptr ||
      stats->summary == nullptr)
    return RBS_ERR_NULL;
  if (!aligned16(stats->centroids) || !aligned16(stats->radii) || !aligned16(stats->beta) ||
      !aligned16(stats->summary))
    return RBS_ERR_ALIGN;
  const int M = blocks_of(shape);
  unsigned char* sum = static_cast<unsigned char*>(stats->summary);
  return finish(rbs::launch_summarize(
      stats->centroids, stats->radii, stats->beta, shape->n_kv_heads, M, reinterpret_cast<_Float16*>(sum),
      reinterpret_cast<float*>(sum + rbs::summary_uplift_offset(shape->n_kv_heads, M)),
      reinterpret_cast<float*>(sum + rbs::summary_cnorm_offset(shape->n_kv_heads, M)),
      static_cast<hipStream_t>(stream)), stream);
}

int rbs_select(const rbs_shape* shape, const void* Q, const rbs_stats* stats, float tau_base, float tau_rescue,
               int32_t n_sink, int32_t n_local, int32_t n_recent, int32_t* counts, int32_t* indices,
               void* stream) {
  int rc = check_shape(shape);
  if (rc != RBS_OK) return rc;
  if (Q == nullptr || counts == nullptr || indices == nullptr || stats == nullptr || stats->summary == nullptr)
    return RBS_ERR_NULL;
  if (!(tau_base >= 0.f && tau_base <= 1.f) || !(tau_rescue >= 0.f && tau_rescue <= 1.f)) return RBS_ERR_ARG;
  if (n_sink < 0 || n_local < 1 || n_recent < 0) return RBS_ERR_ARG;
  if (!aligned16(Q) || !aligned16(counts) || !aligned16(indices) || !aligned16(stats->summary)) return RBS_ERR_ALIGN;
  const int M = blocks_of(shape);
  rbs::Strides st;
  strides_of(shape, &st);
  rbs::SelectArgs a;
  a.Q = static_cast<const uint16_t*>(Q);
  a.q_head = st.q_head;
  a.q_tok = st.q_tok;
  a.n_tokens = shape->n_tokens;
  a.n_q_heads = shape->n_q_heads;
  a.n_kv_heads = shape->n_kv_heads;
  a.block_size = shape->block_size;
  a.n_blocks = M;
  a.cent16 = static_cast<const _Float16*>(stats->summary);
  a.uplift = reinterpret_cast<const float*>(static_cast<const unsigned char*>(stats->summary) +
                                            rbs::summary_uplift_offset(shape->n_kv_heads, M));
  a.cnorm = reinterpret_cast<const float*>(static_cast<const unsigned char*>(stats->summary) +
                                           rbs::summary_cnorm_offset(shape->n_kv_heads, M));
  a.tau_base = tau_base;
  a.tau_rescue = tau_rescue;
  a.n_sink = n_sink;
  a.n_local = n_local;
  a.n_recent = n_recent;
  a.counts = counts;
  a.indices = indices;
  a.capacity = rbs_index_capacity(M);
  rc = check_q_range(Q, st.q_head, st.q_tok, shape->n_q_heads, shape->n_tokens, stream);
  if (rc != RBS_OK) return rc;
  return finish(rbs::launch_select(a, static_cast<hipStream_t>(stream)), stream);
}

int rbs_sparse_prefill(const rbs_shape* shape, const void* Q, const void* K, const void* V, const int32_t* counts,
                       const int32_t* indices, float softmax_scale, void* O, float* lse, void* workspace,
                       void* stream) {
  int rc = check_shape(shape);
  if (rc != RBS_OK) return rc;
  if (Q == nullptr || K == nullptr || V == nullptr || counts == nullptr || indices == nullptr || O == nullptr)
    return RBS_ERR_NULL;
  if (!(softmax_scale == softmax_scale) || isinf(softmax_scale)) return RBS_ERR_ARG;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(counts) || !aligned16(indices) ||
      !aligned16(O) || (lse != nullptr && !aligned16(lse)) || (workspace != nullptr && !aligned16(workspace)))
    return RBS_ERR_ALIGN;
  const int M = blocks_of(shape);
  rbs::AttnArgs a;
  a.Q = static_cast<const uint16_t*>(Q);
  a.K = static_cast<const uint16_t*>(K);
  a.V = static_cast<const uint16_t*>(V);
  strides_of(shape, &a.st);
  a.n_tokens = shape->n_tokens;
  a.n_q_heads = shape->n_q_heads;
  a.n_kv_heads = shape->n_kv_heads;
  a.block_size = shape->block_size;
  a.n_blocks = M;
  a.counts = counts;
  a.indices = indices;
  a.capacity = rbs_index_capacity(M);
  a.scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)shape->head_dim);
  a.O = static_cast<uint16_t*>(O);
  a.lse = lse;
  a.queue = static_cast<int*>(workspace);
  return finish(rbs::launch_attention(a, static_cast<hipStream_t>(stream)), stream);
}

int rbs_sparse_prefill_noalloc(const rbs_shape* shape, const void* Q, const void* K, const void* V,
                               const int32_t* counts, const int32_t* indices, float softmax_scale, void* O,
                               float* lse, void* stream) {
  int rc = check_shape(shape);
  if (rc != RBS_OK) return rc;
  if (Q == nullptr || K == nullptr || V == nullptr || counts == nullptr || indices == nullptr || O == nullptr)
    return RBS_ERR_NULL;
  if (!(softmax_scale == softmax_scale) || isinf(softmax_scale)) return RBS_ERR_ARG;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(counts) || !aligned16(indices) ||
      !aligned16(O) || (lse != nullptr && !aligned16(lse)))
    return RBS_ERR_ALIGN;
  const int M = blocks_of(shape);
  rbs::AttnArgs a;
  a.Q = static_cast<const uint16_t*>(Q);
  a.K = static_cast<const uint16_t*>(K);
  a.V = static_cast<const uint16_t*>(V);
  strides_of(shape, &a.st);
  a.n_tokens = shape->n_tokens;
  a.n_q_heads = shape->n_q_heads;
  a.n_kv_heads = shape->n_kv_heads;
  a.block_size = shape->block_size;
  a.n_blocks = M;
  a.counts = counts;
  a.indices = indices;
  a.capacity = rbs_index_capacity(M);
  a.scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)shape->head_dim);
  a.O = static_cast<uint16_t*>(O);
  a.lse = lse;
  return finish(rbs::launch_attention_noalloc(a, static_cast<hipStream_t>(stream)), stream);
}

int rbs_select_attend(const rbs_shape* shape, const void* Q, const void* K, const void* V, const rbs_stats* stats,
                      float tau_base, float tau_rescue, int32_t n_sink, int32_t n_local, int32_t n_recent,
                      float softmax_scale, int32_t* counts, int32_t* indices, void* O, float* lse, void* workspace,
                      void* stream) {
  int rc = check_shape(shape);
  if (rc != RBS_OK) return rc;
  if (Q == nullptr || K == nullptr || V == nullptr || O == nullptr || counts == nullptr || indices == nullptr ||
      stats == nullptr || stats->summary == nullptr)
    return RBS_ERR_NULL;
  if (!(tau_base >= 0.f && tau_base <= 1.f) || !(tau_rescue >= 0.f && tau_rescue <= 1.f)) return RBS_ERR_ARG;
  if (n_sink < 0 || n_local < 1 || n_recent < 0) return RBS_ERR_ARG;
  if (!(softmax_scale == softmax_scale) || isinf(softmax_scale)) return RBS_ERR_ARG;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O) || !aligned16(counts) ||
      !aligned16(indices) || !aligned16(stats->summary) || (lse != nullptr && !aligned16(lse)) ||
      (workspace != nullptr && !aligned16(workspace)))
    return RBS_ERR_ALIGN;
  const int M = blocks_of(shape);
  rbs::Strides st;
  strides_of(shape, &st);
  rbs::SelectArgs sa;
  sa.Q = static_cast<const uint16_t*>(Q);
  sa.q_head = st.q_head;
  sa.q_tok = st.q_tok;
  sa.n_tokens = shape->n_tokens;
  sa.n_q_heads = shape->n_q_heads;
  sa.n_kv_heads = shape->n_kv_heads;
  sa.block_size = shape->block_size;
  sa.n_blocks = M;
  sa.cent16 = static_cast<const _Float16*>(stats->summary);
  sa.uplift = reinterpret_cast<const float*>(static_cast<const unsigned char*>(stats->summary) +
                                             rbs::summary_uplift_offset(shape->n_kv_heads, M));
  sa.cnorm = reinterpret_cast<const float*>(static_cast<const unsigned char*>(stats->summary) +
                                            rbs::summary_cnorm_offset(shape->n_kv_heads, M));
  sa.tau_base = tau_base;
  sa.tau_rescue = tau_rescue;
  sa.n_sink = n_sink;
  sa.n_local = n_local;
  sa.n_recent = n_recent;
  sa.counts = counts;
  sa.indices = indices;
  sa.capacity = rbs_index_capacity(M);
  rbs::AttnArgs aa;
  aa.Q = sa.Q;
  aa.K = static_cast<const uint16_t*>(K);
  aa.V = static_cast<const uint16_t*>(V);
  aa.st = st;
  aa.n_tokens = shape->n_tokens;
  aa.n_q_heads = shape->n_q_heads;
  aa.n_kv_heads = shape->n_kv_heads;
  aa.block_size = shape->block_size;
  aa.n_blocks = M;
  aa.counts = counts;
  aa.indices = indices;
  aa.capacity = sa.capacity;
  aa.scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)shape->head_dim);
  aa.O = static_cast<uint16_t*>(O);
  aa.lse = lse;
  aa.queue = static_cast<int*>(workspace);
  aa.selected = true;
  rc = check_q_range(Q, st.q_head, st.q_tok, shape->n_q_heads, shape->n_tokens, stream);
  if (rc != RBS_OK) return rc;
  // The two stages' own kernels, one after the other: a kernel that did both
  // kept its selection at the attention's occupancy (2 workgroups per compute
  // unit) and was slower nearly everywhere.  One kernel / two, whole calls: 64K
  // tokens, 64 / 8 heads, B = 128 26.5 / 25.5 ms; B = 64, 32 / 4 heads 8000 tokens
  // 242 / 239 us, 8 / 1 20000 246 / 244; the other way 59084 tokens with one head
  // (selection and attention both a few rows' latency) 174 / 186.
  hipError_t e = rbs::launch_select(sa, static_cast<hipStream_t>(stream));
  if (e == hipSuccess) e = rbs::launch_attention(aa, static_cast<hipStream_t>(stream));
  return finish(e, stream);
}

size_t rbs_box_summary_bytes(const rbs_shape* shape) {
  if (check_shape(shape) != RBS_OK) return 0;
  return 2 * box_half_offset(shape->n_kv_heads, blocks_of(shape));
}

int rbs_block_box(const rbs_shape* shape, const void* K, const rbs_box* box, void* stream) {
  int rc = check_shape(shape);
  if (rc != RBS_OK) return rc;
  if (K == nullptr || box == nullptr || box->center == nullptr || box->half == nullptr || box->summary == nullptr)
    return RBS_ERR_NULL;
  if (!aligned16(K) || !aligned16(box->center) || !aligned16(box->half) || !aligned16(box->summary))
    return RBS_ERR_ALIGN;
  const int M = blocks_of(shape);
  rbs::Strides st;
  strides_of(shape, &st);
  rbs::BoxArgs a;
  a.K = static_cast<const uint16_t*>(K);
  a.kv_head = st.kv_head;
  a.kv_tok = st.kv_tok;
  a.n_tokens = shape->n_tokens;
  a.n_kv_heads = shape->n_kv_heads;
  a.block_size = shape->block_size;
  a.n_blocks = M;
  a.center = box->center;
  a.half = box->half;
  a.center16 = static_cast<_Float16*>(box->summary);
  a.half16 = reinterpret_cast<_Float16*>(static_cast<unsigned char*>(box->summary) +
                                         box_half_offset(shape->n_kv_heads, M));
  return finish(rbs::launch_box(a, static_cast<hipStream_t>(stream)), stream);
}

int rbs_select_variant(const rbs_shape* shape, const void* Q, const rbs_stats* stats, const rbs_box* box,
                       int32_t selector, float param, int32_t n_sink, int32_t n_local, int32_t n_recent,
                       int32_t* counts, int32_t* indices, void* stream) {
  int rc = check_shape(shape);
  if (rc != RBS_OK) return rc;
  if (Q == nullptr || counts == nullptr || indices == nullptr || stats == nullptr || stats->summary == nullptr)
    return RBS_ERR_NULL;
  if (selector != RBS_SELECTOR_CENTROID && selector != RBS_SELECTOR_FULL_L2 && selector != RBS_SELECTOR_BOX)
    return RBS_ERR_ARG;
  if (selector == RBS_SELECTOR_BOX) {
    if (!(param > 0.f && param <= 1.f)) return RBS_ERR_ARG;
    if (box == nullptr || box->summary == nullptr) return RBS_ERR_NULL;
    if (!aligned16(box->summary)) return RBS_ERR_ALIGN;
  } else if (!(param >= 0.f && param <= 1.f)) {
    return RBS_ERR_ARG;
  }
  if (selector == RBS_SELECTOR_FULL_L2) {
    if (stats->radii == nullptr) return RBS_ERR_NULL;
    if (!aligned16(stats->radii)) return RBS_ERR_ALIGN;
  }
  if (n_sink < 0 || n_local < 1 || n_recent < 0) return RBS_ERR_ARG;
  if (!aligned16(Q) || !aligned16(counts) || !aligned16(indices) || !aligned16(stats->summary)) return RBS_ERR_ALIGN;
  const int M = blocks_of(shape);
  rbs::Strides st;
  strides_of(shape, &st);
  rbs::SelectArgs a;
  a.Q = static_cast<const uint16_t*>(Q);
  a.q_head = st.q_head;
  a.q_tok = st.q_tok;
  a.n_tokens = shape->n_tokens;
  a.n_q_heads = shape->n_q_heads;
  a.n_kv_heads = shape->n_kv_heads;
  a.block_size = shape->block_size;
  a.n_blocks = M;
  a.mode = selector;  // RBS_SELECTOR_* equals the kernel's SelectMode
  if (selector == RBS_SELECTOR_BOX) {
    a.cent16 = static_cast<const _Float16*>(box->summary);
    a.half16 = reinterpret_cast<const _Float16*>(static_cast<const unsigned char*>(box->summary) +
                                                 box_half_offset(shape->n_kv_heads, M));
    a.budget = param;
    a.tau_base = a.tau_rescue = 1.f;  // unused
  } else {
    a.cent16 = static_cast<const _Float16*>(stats->summary);
    a.cnorm = reinterpret_cast<const float*>(static_cast<const unsigned char*>(stats->summary) +
                                             rbs::summary_cnorm_offset(shape->n_kv_heads, M));
    a.tau_base = a.tau_rescue = param;
  }
  a.uplift = nullptr;
  a.radii = stats->radii;
  a.n_sink = n_sink;
  a.n_local = n_local;
  a.n_recent = n_recent;
  a.counts = counts;
  a.indices = indices;
  a.capacity = rbs_index_capacity(M);
  rc = check_q_range(Q, st.q_head, st.q_tok, shape->n_q_heads, shape->n_tokens, stream);
  if (rc != RBS_OK) return rc;
  return finish(rbs::launch_select(a, static_cast<hipStream_t>(stream)), stream);
}

int rbs_dense_indices(const rbs_shape* shape, int32_t* counts, int32_t* indices, void* stream) {
  int rc = check_shape(shape);
  if (rc != RBS_OK) return rc;
  if (counts == nullptr || indices == nullptr) return RBS_ERR_NULL;
  if (!aligned16(counts) || !aligned16(indices)) return RBS_ERR_ALIGN;
  const int M = blocks_of(shape);
  return finish(rbs::launch_dense_indices(shape->n_q_heads, M, rbs_index_capacity(M), counts, indices,
                                            static_cast<hipStream_t>(stream)), stream);
}

int32_t rbs_varlen_blocks(const rbs_shape* shape, const rbs_batch* batch) {
  rbs::SeqTable t;
  return check_batch(shape, batch, &t) == RBS_OK ? t.blk[t.n] : 0;
}

int64_t rbs_varlen_index_capacity(const rbs_shape* shape, const rbs_batch* batch) {
  rbs::SeqTable t;
  return check_batch(shape, batch, &t) == RBS_OK ? t.cap[t.n] : 0;
}

size_t rbs_varlen_summary_bytes(const rbs_shape* shape, const rbs_batch* batch) {
  rbs::SeqTable t;
  if (check_batch(shape, batch, &t) != RBS_OK) return 0;
  return rbs::summary_bytes(shape->n_kv_heads, t.blk[t.n]);
}

int rbs_block_stats_varlen(const rbs_shape* shape, const rbs_batch* batch, const void* K, const rbs_stats* stats,
                           void* stream) {
  rbs::SeqTable t;
  int rc = check_batch(shape, batch, &t);
  if (rc != RBS_OK) return rc;
  if (K == nullptr) return RBS_ERR_NULL;
  if ((rc = check_stats_ptrs(stats)) != RBS_OK) return rc;
  if (!aligned16(K)) return RBS_ERR_ALIGN;
  const int M = t.blk[t.n];
  rbs::Strides st;
  strides_of(shape, &st);
  rbs::StatsArgs a;
  a.K = static_cast<const uint16_t*>(K);
  a.kv_head = st.kv_head;
  a.kv_tok = st.kv_tok;
  a.n_tokens = shape->n_tokens;
  a.n_kv_heads = shape->n_kv_heads;
  a.block_size = shape->block_size;
  a.n_blocks = M;
  a.centroids = stats->centroids;
  a.radii = stats->radii;
  a.beta = stats->beta;
  a.quantiles = stats->quantiles;
  a.cent16 = static_cast<_Float16*>(stats->summary);
  a.uplift = reinterpret_cast<float*>(static_cast<unsigned char*>(stats->summary) +
                                      rbs::summary_uplift_offset(shape->n_kv_heads, M));
  a.cnorm = reinterpret_cast<float*>(static_cast<unsigned char*>(stats->summary) +
                                     rbs::summary_cnorm_offset(shape->n_kv_heads, M));
  return finish(rbs::launch_stats_varlen(a, t, static_cast<hipStream_t>(stream)), stream);
}

int rbs_select_varlen(const rbs_shape* shape, const rbs_batch* batch, const void* Q, const rbs_stats* stats,
                      float tau_base, float tau_rescue, int32_t n_sink, int32_t n_local, int32_t n_recent,
                      int32_t* counts, int32_t* indices, void* stream) {
  rbs::SeqTable t;
  int rc = check_batch(shape, batch, &t);
  if (rc != RBS_OK) return rc;
  if (Q == nullptr || counts == nullptr || indices == nullptr || stats == nullptr || stats->summary == nullptr)
    return RBS_ERR_NULL;
  if (!(tau_base >= 0.f && tau_base <= 1.f) || !(tau_rescue >= 0.f && tau_rescue <= 1.f)) return RBS_ERR_ARG;
  if (n_sink < 0 || n_local < 1 || n_recent < 0) return RBS_ERR_ARG;
  if (!aligned16(Q) || !aligned16(counts) || !aligned16(indices) || !aligned16(stats->summary)) return RBS_ERR_ALIGN;
  const int M = t.blk[t.n];
  rbs::Strides st;
  strides_of(shape, &st);
  rbs::SelectArgs a;
  a.Q = static_cast<const uint16_t*>(Q);
  a.q_head = st.q_head;
  a.q_tok = st.q_tok;
  a.n_tokens = shape->n_tokens;
  a.n_q_heads = shape->n_q_heads;
  a.n_kv_heads = shape->n_kv_heads;
  a.block_size = shape->block_size;
  a.n_blocks = M;
  a.cent16 = static_cast<const _Float16*>(stats->summary);
  a.uplift = reinterpret_cast<const float*>(static_cast<const unsigned char*>(stats->summary) +
                                            rbs::summary_uplift_offset(shape->n_kv_heads, M));
  a.cnorm = reinterpret_cast<const float*>(static_cast<const unsigned char*>(stats->summary) +
                                           rbs::summary_cnorm_offset(shape->n_kv_heads, M));
  a.tau_base = tau_base;
  a.tau_rescue = tau_rescue;
  a.n_sink = n_sink;
  a.n_local = n_local;
  a.n_recent = n_recent;
  a.counts = counts;
  a.indices = indices;
  a.capacity = t.cap[t.n];
  rc = check_q_range(Q, st.q_head, st.q_tok, shape->n_q_heads, shape->n_tokens, stream);
  if (rc != RBS_OK) return rc;
  return finish(rbs::launch_select_varlen(a, t, static_cast<hipStream_t>(stream)), stream);
}

int rbs_sparse_prefill_varlen(const rbs_shape* shape, const rbs_batch* batch, const void* Q, const void* K,
                              const void* V, const int32_t* counts, const int32_t* indices, float softmax_scale,
                              void* O, float* lse, void* workspace, void* stream) {
  rbs::SeqTable t;
  int rc = check_batch(shape, batch, &t);
  if (rc != RBS_OK) return rc;
  if (Q == nullptr || K == nullptr || V == nullptr || counts == nullptr || indices == nullptr || O == nullptr)
    return RBS_ERR_NULL;
  if (!(softmax_scale == softmax_scale) || isinf(softmax_scale)) return RBS_ERR_ARG;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(counts) || !aligned16(indices) ||
      !aligned16(O) || (lse != nullptr && !aligned16(lse)) || (workspace != nullptr && !aligned16(workspace)))
    return RBS_ERR_ALIGN;
  rbs::AttnArgs a;
  a.Q = static_cast<const uint16_t*>(Q);
  a.K = static_cast<const uint16_t*>(K);
  a.V = static_cast<const uint16_t*>(V);
  strides_of(shape, &a.st);
  a.n_tokens = shape->n_tokens;
  a.n_q_heads = shape->n_q_heads;
  a.n_kv_heads = shape->n_kv_heads;
  a.block_size = shape->block_size;
  a.n_blocks = t.blk[t.n];
  a.counts = counts;
  a.indices = indices;
  a.capacity = t.cap[t.n];
  a.scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)shape->head_dim);
  a.O = static_cast<uint16_t*>(O);
  a.lse = lse;
  a.queue = static_cast<int*>(workspace);
  return finish(rbs::launch_attention_varlen(a, t, static_cast<hipStream_t>(stream)), stream);
}

int rbs_dense_indices_varlen(const rbs_shape* shape, const rbs_batch* batch, int32_t* counts, int32_t* indices,
                             void* stream) {
  rbs::SeqTable t;
  int rc = check_batch(shape, batch, &t);
  if (rc != RBS_OK) return rc;
  if (counts == nullptr || indices == nullptr) return RBS_ERR_NULL;
  if (!aligned16(counts) || !aligned16(indices)) return RBS_ERR_ALIGN;
  return finish(
      rbs::launch_dense_indices_varlen(shape->n_q_heads, t, counts, indices, static_cast<hipStream_t>(stream)), stream);
}

size_t rbs_fp8_vt_bytes(const rbs_shape* shape) {
  if (check_shape(shape) != RBS_OK) return 0;
  return (size_t)shape->n_kv_heads * blocks_of(shape) * 128 * shape->block_size;
}

int rbs_fp8_amax(const rbs_shape* shape, const void* Q, const void* K, const void* V, float* amax, void* stream) {
  int rc = check_shape(shape);
  if (rc != RBS_OK) return rc;
  if (Q == nullptr || K == nullptr || V == nullptr || amax == nullptr) return RBS_ERR_NULL;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(amax)) return RBS_ERR_ALIGN;
  rbs::Strides st;
  strides_of(shape, &st);
  return finish(rbs::launch_fp8_amax(static_cast<const uint16_t*>(Q), static_cast<const uint16_t*>(K),
                                       static_cast<const uint16_t*>(V), st, shape->n_tokens, shape->n_q_heads,
                                       shape->n_kv_heads, amax, static_cast<hipStream_t>(stream)), stream);
}

int rbs_fp8_pack(const rbs_shape* shape, const void* Q, const void* K, const void* V, const float* amax, void* Q8,
                 void* K8, void* V8t, void* stream) {
  int rc = check_shape(shape);
  if (rc != RBS_OK) return rc;
  if (Q == nullptr || K == nullptr || V == nullptr || amax == nullptr || Q8 == nullptr || K8 == nullptr ||
      V8t == nullptr)
    return RBS_ERR_NULL;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(amax) || !aligned16(Q8) || !aligned16(K8) ||
      !aligned16(V8t))
    return RBS_ERR_ALIGN;
  rbs::Strides st;
  strides_of(shape, &st);
  return finish(rbs::launch_fp8_pack(static_cast<const uint16_t*>(Q), static_cast<const uint16_t*>(K),
                                       static_cast<const uint16_t*>(V), st, shape->n_tokens, shape->n_q_heads,
                                       shape->n_kv_heads, shape->block_size, blocks_of(shape), amax,
                                       static_cast<uint8_t*>(Q8),
                                       static_cast<uint8_t*>(K8), static_cast<uint8_t*>(V8t),
                                       static_cast<hipStream_t>(stream)), stream);
}

int rbs_sparse_prefill_fp8(const rbs_shape* shape, const void* Q8, const void* K8, const void* V8t,
                           const float* amax, const int32_t* counts, const int32_t* indices, float softmax_scale,
                           void* O, float* lse, void* workspace, void* stream) {
  int rc = check_shape(shape);
  if (rc != RBS_OK) return rc;
  if (Q8 == nullptr || K8 == nullptr || V8t == nullptr || amax == nullptr || counts == nullptr ||
      indices == nullptr || O == nullptr)
    return RBS_ERR_NULL;
  if (!(softmax_scale == softmax_scale) || isinf(softmax_scale)) return RBS_ERR_ARG;
  if (!aligned16(Q8) || !aligned16(K8) || !aligned16(V8t) || !aligned16(amax) || !aligned16(counts) ||
      !aligned16(indices) || !aligned16(O) || (lse != nullptr && !aligned16(lse)) ||
      (workspace != nullptr && !aligned16(workspace)))
    return RBS_ERR_ALIGN;
  const int M = blocks_of(shape);
  const float scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)shape->head_dim);
  rbs::Strides st;
  strides_of(shape, &st);
  return finish(rbs::launch_attention_fp8(
      static_cast<const uint8_t*>(Q8), static_cast<const uint8_t*>(K8), static_cast<const uint8_t*>(V8t), amax,
      shape->n_tokens, shape->n_q_heads, shape->n_kv_heads, shape->block_size, M, counts, indices,
      rbs_index_capacity(M), scale, static_cast<uint16_t*>(O), st.q_head, st.q_tok, lse,
      static_cast<int*>(workspace), static_cast<hipStream_t>(stream)), stream);
}

int rbs_pages_extend(const rbs_pages* pages, const int32_t* seq_lens, const int32_t* new_tokens,
                     const int32_t* n_free, int32_t max_tokens, int32_t* seq_lens_out, int32_t* n_free_out,
                     int32_t* cu_tokens, int32_t* positions, int32_t* slots, int32_t* status, void* stream) {
  int shift;
  int rc = check_pages(pages, &shift);
  if (rc != RBS_OK) return rc;
  if (max_tokens < 1 || max_tokens > RBS_MAX_NEW_TOKENS) return RBS_ERR_SHAPE;
  if (seq_lens == nullptr || n_free == nullptr || seq_lens_out == nullptr || n_free_out == nullptr ||
      cu_tokens == nullptr || positions == nullptr || slots == nullptr || status == nullptr)
    return RBS_ERR_NULL;
  if (!aligned16(seq_lens) || (new_tokens != nullptr && !aligned16(new_tokens)) || !aligned16(n_free) ||
      !aligned16(seq_lens_out) || !aligned16(n_free_out) || !aligned16(cu_tokens) || !aligned16(positions) ||
      !aligned16(slots) || !aligned16(status))
    return RBS_ERR_ALIGN;
  rbs::PagesArgs a;
  a.n_rows = pages->n_rows;
  a.max_pages = pages->max_pages;
  a.n_pages = pages->n_pages;
  a.page_shift = shift;
  a.page_table = pages->page_table;
  a.free_pages = pages->free_pages;
  a.seq_lens = seq_lens;
  a.new_tokens = new_tokens;
  a.n_free = n_free;
  a.max_tokens = max_tokens;
  a.seq_lens_out = seq_lens_out;
  a.n_free_out = n_free_out;
  a.cu_tokens = cu_tokens;
  a.positions = positions;
  a.slots = slots;
  a.status = status;
  return finish(rbs::launch_pages_extend(a, static_cast<hipStream_t>(stream)), stream);
}

int rbs_pages_release(const rbs_pages* pages, const int32_t* released, int32_t* seq_lens, int32_t* n_free,
                      int32_t* status, void* stream) {
  int shift;
  int rc = check_pages(pages, &shift);
  if (rc != RBS_OK) return rc;
  if (released == nullptr || seq_lens == nullptr || n_free == nullptr || status == nullptr) return RBS_ERR_NULL;
  if (!aligned16(released) || !aligned16(seq_lens) || !aligned16(n_free) || !aligned16(status)) return RBS_ERR_ALIGN;
  return finish(rbs::launch_pages_release(pages->n_rows, pages->max_pages, pages->n_pages, shift, pages->page_table,
                                          pages->free_pages, released, seq_lens, n_free, status,
                                          static_cast<hipStream_t>(stream)), stream);
}

int rbs_qk_norm_rope(const rbs_shape* in, const rbs_shape* out, const rbs_rope* rope, const void* Q, const void* K,
                     const void* V, const int32_t* positions, void* Q_out, void* K_out, const rbs_cache* cache,
                     const int32_t* slots, void* stream) {
  int rc = check_heads(in, RBS_MAX_NEW_TOKENS);
  if (rc != RBS_OK) return rc;
  rbs::RopeArgs a{};
  if ((rc = strides_of(in, &a.in)) != RBS_OK) return rc;
  a.out = a.in;
  if (out != nullptr) {
    if (out->n_tokens != in->n_tokens || out->n_q_heads != in->n_q_heads || out->n_kv_heads != in->n_kv_heads ||
        out->head_dim != in->head_dim)
      return RBS_ERR_SHAPE;
    if ((rc = strides_of(out, &a.out)) != RBS_OK) return rc;
  }
  if (rope == nullptr || Q == nullptr || K == nullptr || positions == nullptr || Q_out == nullptr)
    return RBS_ERR_NULL;
  if (rope->rot_dim < 0 || rope->rot_dim > 128 || rope->rot_dim % 8 != 0) return RBS_ERR_UNSUPPORTED;
  if (!(rope->eps >= 0.f) || isinf(rope->eps) || !(rope->factor == rope->factor) || isinf(rope->factor))
    return RBS_ERR_ARG;
  if (rope->rot_dim > 0 && rope->inv_freq == nullptr) return RBS_ERR_NULL;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(positions) || !aligned16(Q_out) || !aligned16(K_out) ||
      !aligned16(rope->q_weight) || !aligned16(rope->k_weight) || !aligned16(rope->inv_freq))
    return RBS_ERR_ALIGN;
  // In place only row by row: the same pointer needs the same strides.
  if ((Q_out == Q && (a.out.q_head != a.in.q_head || a.out.q_tok != a.in.q_tok)) ||
      (K_out == K && (a.out.kv_head != a.in.kv_head || a.out.kv_tok != a.in.kv_tok)))
    return RBS_ERR_SHAPE;
  if (cache != nullptr) {
    if ((rc = check_cache(cache, &a.cache)) != RBS_OK) return rc;
    if (cache->n_kv_heads != in->n_kv_heads) return RBS_ERR_SHAPE;
    if (V == nullptr || slots == nullptr) return RBS_ERR_NULL;
    if (!aligned16(V) || !aligned16(slots)) return RBS_ERR_ALIGN;
    a.cached = true;
  }
  a.Q = static_cast<const uint16_t*>(Q);
  a.K = static_cast<const uint16_t*>(K);
  a.V = static_cast<const uint16_t*>(V);
  a.n_tokens = in->n_tokens;
  a.n_q_heads = in->n_q_heads;
  a.n_kv_heads = in->n_kv_heads;
  a.q_weight = static_cast<const uint16_t*>(rope->q_weight);
  a.k_weight = static_cast<const uint16_t*>(rope->k_weight);
  a.inv_freq = rope->inv_freq;
  a.rot_dim = rope->rot_dim;
  a.interleaved = rope->interleaved != 0;
  a.eps = rope->eps;
  a.factor = rope->factor;
  a.positions = positions;
  a.slots = slots;
  a.Q_out = static_cast<uint16_t*>(Q_out);
  a.K_out = static_cast<uint16_t*>(K_out);
  return finish(rbs::launch_qk_norm_rope(a, static_cast<hipStream_t>(stream)), stream);
}

size_t rbs_decode_workspace_bytes(void) { return rbs::decode_workspace_bytes(); }

// packed: rows take their tokens by cu_tokens; otherwise the shape's tokens are the rows.
static int paged_decode(const rbs_shape* shape, const rbs_cache* cache, const void* Q, bool packed,
                        const int32_t* cu_tokens, int32_t n_rows, const int32_t* page_table, int32_t max_pages,
                        const int32_t* seq_lens, float softmax_scale, void* O, float* lse, void* workspace,
                        void* stream) {
  static_assert(RBS_MAX_ROWS == rbs::kMaxRows, "rows of a page table");
  int rc = check_heads(shape, packed ? RBS_MAX_NEW_TOKENS : RBS_MAX_ROWS);
  if (rc != RBS_OK) return rc;
  if (!packed) n_rows = shape->n_tokens;
  if (n_rows < 1 || n_rows > RBS_MAX_ROWS) return RBS_ERR_SHAPE;
  rbs::DecodeArgs a{};
  if ((rc = resolve_strides(shape->q_stride_head, shape->q_stride_tok, shape->n_q_heads, shape->n_tokens, &a.q_head,
                            &a.q_tok)) != RBS_OK)
    return rc;
  if ((rc = check_cache(cache, &a.cache)) != RBS_OK) return rc;
  if (cache->n_kv_heads != shape->n_kv_heads || max_pages < 1 || max_pages > (INT32_MAX >> a.cache.page_shift))
    return RBS_ERR_SHAPE;
  // The shares of all rows are counted in 32 bits.
  if (n_rows * ((((int64_t)max_pages << a.cache.page_shift) >> 5) + 8) > INT32_MAX) return RBS_ERR_SHAPE;
  if (Q == nullptr || page_table == nullptr || seq_lens == nullptr || O == nullptr || workspace == nullptr ||
      (packed && cu_tokens == nullptr))
    return RBS_ERR_NULL;
  if (!(softmax_scale == softmax_scale) || isinf(softmax_scale)) return RBS_ERR_ARG;
  if (!aligned16(Q) || !aligned16(page_table) || !aligned16(seq_lens) || !aligned16(O) || !aligned16(lse) ||
      !aligned16(workspace) || !aligned16(cu_tokens))
    return RBS_ERR_ALIGN;
  a.Q = static_cast<const uint16_t*>(Q);
  a.n_tokens = shape->n_tokens;
  a.n_rows = n_rows;
  a.n_q_heads = shape->n_q_heads;
  a.n_kv_heads = shape->n_kv_heads;
  a.page_table = page_table;
  a.max_pages = max_pages;
  a.seq_lens = seq_lens;
  a.cu_tokens = packed ? cu_tokens : nullptr;
  a.scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)shape->head_dim);
  a.O = static_cast<uint16_t*>(O);
  a.lse = lse;
  a.workspace = static_cast<float*>(workspace);
  return finish(rbs::launch_paged_decode(a, static_cast<hipStream_t>(stream)), stream);
}

int rbs_paged_decode(const rbs_shape* shape, const rbs_cache* cache, const void* Q, const int32_t* page_table,
                     int32_t max_pages, const int32_t* seq_lens, float softmax_scale, void* O, float* lse,
                     void* workspace, void* stream) {
  return paged_decode(shape, cache, Q, false, nullptr, 0, page_table, max_pages, seq_lens, softmax_scale, O, lse,
                      workspace, stream);
}

int rbs_paged_decode_packed(const rbs_shape* shape, const rbs_cache* cache, const void* Q, const int32_t* cu_tokens,
                            int32_t n_rows, const int32_t* page_table, int32_t max_pages, const int32_t* seq_lens,
                            float softmax_scale, void* O, float* lse, void* workspace, void* stream) {
  return paged_decode(shape, cache, Q, true, cu_tokens, n_rows, page_table, max_pages, seq_lens, softmax_scale, O,
                      lse, workspace, stream);
}

const char* rbs_status_str(int status) {
  switch (status) {
    case RBS_OK: return "ok";
    case RBS_ERR_NULL: return "null pointer argument";
    case RBS_ERR_SHAPE: return "invalid shape (token/head counts, head ratio, size limits or strides)";
    case RBS_ERR_UNSUPPORTED: return "unsupported head_dim or block_size (need d = 128, B in {64, 128, 256})";
    case RBS_ERR_ARG: return "invalid argument (threshold outside [0, 1], window < 1, bad scale)";
    case RBS_ERR_ALIGN: return "device pointer not 16-byte aligned";
    case RBS_ERR_HIP: return "HIP runtime rejected a kernel launch (in debug mode: or a kernel failed)";
    case RBS_ERR_RANGE: return "a query element is beyond the selector's f16 range (+-65504) or not finite";
    default: return "unknown status";
  }
}

int rbs_set_debug(int on) {
  const int prev = debug_on() ? 1 : 0;
  g_debug.store(on != 0 ? 1 : 0, std::memory_order_relaxed);
  return prev;
}

}  // extern "C"
