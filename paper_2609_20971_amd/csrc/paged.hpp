// The calls over a paged key-value cache (paged.hip, cache.hip, decode.hip,
// prefill.hip): what api.hip hands them, arguments validated, and what they share on
// the device.
#pragma once

#include "rbs_device.hpp"
#include "rbs_launch.hpp"

namespace rbs {

constexpr int kCacheBf16 = 0, kCacheFp8 = 1, kCacheFp4 = 4;  // RBS_CACHE_*

// K and V of a paged cache: element (page, head, place, j) at page * page + ...
struct CacheView {
  void* K;
  void* V;
  const float* amax;  // FP8 only
  int64_t page, head, tok;
  int n_pages, page_shift;
  int format;
  void* K_scale;      // FP4 only: that of element x (a multiple of 32) at byte x / 32
  void* V_scale;
};

struct PagesArgs {
  int n_rows, max_pages, n_pages, page_shift;
  int32_t* page_table;
  const int32_t* free_pages;
  const int32_t* seq_lens;
  const int32_t* new_tokens;  // null: one each
  const int32_t* n_free;
  int max_tokens;
  int32_t* seq_lens_out;
  int32_t* n_free_out;
  int32_t* cu_tokens;
  int32_t* positions;
  int32_t* slots;
  int32_t* status;
};

struct RopeArgs {
  const uint16_t* Q;
  const uint16_t* K;
  const uint16_t* V;
  Strides in, out;  // out.kv_*: K_out
  int n_tokens, n_q_heads, n_kv_heads;
  const uint16_t* q_weight;
  const uint16_t* k_weight;
  const float* inv_freq;
  int rot_dim;
  bool interleaved;
  float eps, factor;
  const int32_t* positions;
  const int32_t* slots;
  uint16_t* Q_out;
  uint16_t* K_out;  // null: not kept
  bool cached;
  CacheView cache;
};

// rbs_cache_write and rbs_cache_read: rows between bf16 tensors and a cache.
struct MoveArgs {
  uint16_t* K;  // (read by the one, written by the other)
  uint16_t* V;
  int64_t k_head, k_tok, v_head, v_tok;
  int n_tokens, n_kv_heads;
  CacheView cache;
  const int32_t* slots;      // write: of each token
  const int32_t* cu_tokens;  // read: rows' packed tokens,
  const int32_t* starts;     // and the position of each row's first one (null: 0)
  int n_rows, max_pages;
  const int32_t* page_table;
};

struct DecodeArgs {
  const uint16_t* Q;
  int64_t q_head, q_tok;  // Q and O
  int n_tokens;           // of Q, O and lse
  int n_rows, n_q_heads, n_kv_heads;
  CacheView cache;
  const int32_t* page_table;
  int max_pages;
  const int32_t* seq_lens;
  const int32_t* cu_tokens;  // row s's token is cu_tokens[s + 1] - 1; null: s
  float scale;
  uint16_t* O;
  float* lse;
  float* workspace;
};

// rbs_paged_prefill: as above, every new token of a row a query.
struct PrefillArgs {
  const uint16_t* Q;
  int64_t q_head, q_tok;  // Q and O
  int n_tokens;           // of Q, O and lse
  int n_rows, n_q_heads, n_kv_heads;
  CacheView cache;
  const int32_t* page_table;
  int max_pages;
  const int32_t* seq_lens;
  const int32_t* cu_tokens;
  float scale;
  uint16_t* O;
  float* lse;
  float* workspace;
};

constexpr int kMaxRows = 4096;  // rows of a page table

hipError_t launch_pages_extend(const PagesArgs& a, hipStream_t s);
hipError_t launch_pages_release(int n_rows, int max_pages, int n_pages, int page_shift, const int32_t* page_table,
                                int32_t* free_pages, const int32_t* released, int32_t* seq_lens, int32_t* n_free,
                                int32_t* status, hipStream_t s);
hipError_t launch_qk_norm_rope(const RopeArgs& a, hipStream_t s);
hipError_t launch_cache_write(const MoveArgs& a, hipStream_t s);
hipError_t launch_cache_read(const MoveArgs& a, hipStream_t s);
size_t decode_workspace_bytes();
hipError_t launch_paged_decode(const DecodeArgs& a, hipStream_t s);
size_t prefill_workspace_bytes();
hipError_t launch_paged_prefill(const PrefillArgs& a, hipStream_t s);

// x combined over the lanes up to and with this one (op: associative, 0 its
// neutral element): within each row of 16 lanes, then the last lane of row 0 (2)
// onto row 1 (3), then that of the first two rows onto the others.  A lane or row
// with no source takes 0.
template <typename Op>
__device__ __forceinline__ int wave_scan(int x, Op op) {
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false));  // row_shr 1
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false));  // row_shr 2
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false));  // row_shr 4
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false));  // row_shr 8
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));  // row_bcast 15
  return op(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));  // row_bcast 31
}

typedef __bf16 bf16x2 __attribute__((__vector_size__(2 * sizeof(__bf16))));

// The scale byte of 32 elements whose largest magnitude has these 15 bits of bf16:
// 2^(byte - 127) is the least power of two (from 2^-126) that takes it under 7, so
// that it rounds to 6 or less and no element is off by more than half a step of the
// codes' largest binade (7 / 4 of a power of two is where the 32 carries into the
// exponent).  255: a NaN or an infinity among them.  (From 7 / 4 2^127 on the nearest code
// stands for 2^128, which bf16 and fp32 have as infinity.)
__device__ __forceinline__ uint32_t fp4_scale(uint32_t top) {
  return (top >> 7) == 255u ? 255u : (uint32_t)max((int)((top + 32u) >> 7) - 2, 1);
}

// E2M1 codes (nearest even) of 8 bf16 over the scale; 0 under a scale of 255.
__device__ __forceinline__ uint32_t pack_e2m1(const uint32_t* pairs, uint32_t scale) {
  const float f = __uint_as_float(scale << 23);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, pairs[0]), f, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, pairs[1]), f, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, pairs[2]), f, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, pairs[3]), f, 3);
  return scale == 255u ? 0u : w;
}

// bf16 of eight E2M1 codes times 2^(scale - 127), scale in bits 23 .. 30 (255: NaN); exact.
__device__ __forceinline__ uint4 widen_e2m1(uint32_t codes, uint32_t scale) {
  const float f = __uint_as_float(scale);
  return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, f, 0)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, f, 1)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, f, 2)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, f, 3)));
}

// E4M3 codes of four values times scale, saturating at +-448 (NaN stays NaN).
__device__ __forceinline__ uint32_t pack_e4m3(const float* x, float scale) {
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[i] = x[i] * scale;
    y[i] = y[i] > 448.f ? 448.f : y[i] < -448.f ? -448.f : y[i];
  }
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
}

// kWords words between memory and registers; kOnce: with no place in the caches.
template <int kWords, bool kOnce>
__device__ __forceinline__ void load_words(const void* p, uint32_t* w) {
  typedef uint32_t Vec __attribute__((ext_vector_type(kWords)));
  const Vec v = kOnce ? __builtin_nontemporal_load(static_cast<const Vec*>(p)) : *static_cast<const Vec*>(p);
#pragma unroll
  for (int i = 0; i < kWords; ++i) w[i] = v[i];
}
template <int kWords, bool kOnce>
__device__ __forceinline__ void store_words(void* p, const uint32_t* w) {
  typedef uint32_t Vec __attribute__((ext_vector_type(kWords)));
  Vec v;
#pragma unroll
  for (int i = 0; i < kWords; ++i) v[i] = w[i];
  if (kOnce) __builtin_nontemporal_store(v, static_cast<Vec*>(p));
  else *static_cast<Vec*>(p) = v;
}

// Two fp32 to bf16 (nearest even) in one word.
__device__ __forceinline__ uint32_t two_bf16(float a, float b) {
  const bf16x2 v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, v);
}

}  // namespace rbs
