// The calls over a paged key-value cache (paged.hip, decode.hip): what api.hip
// hands them, arguments validated, and what the two share on the device.
#pragma once

#include "rbs_device.hpp"
#include "rbs_launch.hpp"

namespace rbs {

// K and V of a paged cache: element (page, head, place, j) at page * page + ...
struct CacheView {
  void* K;
  void* V;
  const float* amax;  // null: bf16
  int64_t page, head, tok;
  int n_pages, page_shift;
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

constexpr int kMaxRows = 4096;  // rows of a page table

hipError_t launch_pages_extend(const PagesArgs& a, hipStream_t s);
hipError_t launch_pages_release(int n_rows, int max_pages, int n_pages, int page_shift, const int32_t* page_table,
                                int32_t* free_pages, const int32_t* released, int32_t* seq_lens, int32_t* n_free,
                                int32_t* status, hipStream_t s);
hipError_t launch_qk_norm_rope(const RopeArgs& a, hipStream_t s);
size_t decode_workspace_bytes();
hipError_t launch_paged_decode(const DecodeArgs& a, hipStream_t s);

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

// Two fp32 to bf16 (nearest even) in one word.
__device__ __forceinline__ uint32_t two_bf16(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((__vector_size__(2 * sizeof(__bf16))));
  const bf16x2 v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, v);
}

}  // namespace rbs
