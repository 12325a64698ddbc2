// Around a paged key-value cache: pages and slots of a batch's new tokens, pages
// given back, and queries and keys normed, rotated and put into the cache.
#include "../../include/rbs.h"
#include "rbs_device.hpp"
#include "rbs_launch.hpp"

namespace rbs {

// ------------------------------------------------------------------ pages

constexpr int kPageThreads = 1024;
constexpr int kFillTokens = 4 * kPageThreads;  // tokens (and new pages) of one workgroup
constexpr int kMost = 1 << 29;                 // sums stop here, past every limit that they are compared with

__device__ __forceinline__ int capped_add(int a, int b) { return min(a + b, kMost); }  // a, b in 0 .. kMost

// Sums of two counts over the threads before this one, and over all of them.
// Capped addition of nonnegative numbers is associative, so that the order of
// the partial sums does not matter.
__device__ __forceinline__ void scan_pair(int a, int b, int* sums, int& a_before, int& b_before, int& a_all,
                                          int& b_all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int x = a, y = b;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int u = __shfl_up(x, d), v = __shfl_up(y, d);
    if (lane >= d) {
      x = capped_add(x, u);
      y = capped_add(y, v);
    }
  }
  constexpr int kWaves = kPageThreads / 64;
  if (lane == 63) {
    sums[wave] = x;
    sums[kWaves + wave] = y;
  }
  const int px = __shfl_up(x, 1), py = __shfl_up(y, 1);
  __syncthreads();
  a_before = lane == 0 ? 0 : px;
  b_before = lane == 0 ? 0 : py;
  a_all = b_all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w == wave) {
      a_before = capped_add(a_before, a_all);
      b_before = capped_add(b_before, b_all);
    }
    a_all = capped_add(a_all, sums[w]);
    b_all = capped_add(b_all, sums[kWaves + w]);
  }
}

// Every workgroup sums the rows' counts for itself (n_rows numbers that the L2
// holds), then fills its share of the tokens and new pages: one launch, and no
// table of sums between two.  The state (lengths, n_free, offsets, status) is
// workgroup 0's, where `state` is set.  Bound by latency: three dependent loads
// and a scan.
__global__ __launch_bounds__(kPageThreads) void pages_extend_kernel(PagesArgs a, bool fill, bool state) {
  __shared__ int sums[2 * kPageThreads / 64];
  __shared__ int first_token[kMaxRows + 1], first_page[kMaxRows + 1], length[kMaxRows];
  const int t = threadIdx.x, shift = a.page_shift, places = (1 << shift) - 1;
  const int per = (a.n_rows + kPageThreads - 1) / kPageThreads;  // rows per thread, 1 .. 4
  const int row0 = t * per;
  const int n_free = *a.n_free;
  int add[kMaxRows / kPageThreads], need[kMaxRows / kPageThreads];
  int tokens = 0, pages = 0;
  bool too_long = false;
#pragma unroll
  for (int i = 0; i < kMaxRows / kPageThreads; ++i) {
    add[i] = need[i] = 0;
    const int row = row0 + i;
    if (i < per && row < a.n_rows) {
      const int len = a.seq_lens[row];
      length[row] = len;
      if (len >= 0) {
        const int more = a.new_tokens != nullptr ? max(a.new_tokens[row], 0) : 1;
        const int64_t held = ((int64_t)len + places) >> shift;
        const int64_t after = ((int64_t)len + more + places) >> shift;
        too_long |= after > a.max_pages;
        add[i] = min(more, kMost);
        need[i] = (int)(after - held);  // < 2^28
      }
    }
    tokens = capped_add(tokens, add[i]);
    pages = capped_add(pages, need[i]);
  }
  int token, page, all_tokens, all_pages;
  scan_pair(tokens, pages, sums, token, page, all_tokens, all_pages);
#pragma unroll
  for (int i = 0; i < kMaxRows / kPageThreads; ++i) {
    const int row = row0 + i;
    if (i < per && row < a.n_rows) {
      first_token[row] = token;
      first_page[row] = page;
      token = capped_add(token, add[i]);
      page = capped_add(page, need[i]);
    }
  }
  if (t == 0) {
    first_token[a.n_rows] = all_tokens;
    first_page[a.n_rows] = all_pages;
  }
  const int status = (all_pages > max(n_free, 0) ? RBS_PAGES_FEW : 0) | (__syncthreads_or(too_long) ? RBS_PAGES_ROW : 0) |
                     (all_tokens > a.max_tokens ? RBS_PAGES_TOKENS : 0) |
                     (n_free < 0 || n_free > a.n_pages ? RBS_PAGES_STACK : 0);
  const bool ok = status == 0;

  if (fill) {
    const int begin = blockIdx.x * kFillTokens;
    if (ok) {
      for (int k = begin + t; k < min(begin + kFillTokens, all_pages); k += kPageThreads) {
        const int row = seq_of(first_page, a.n_rows, k);
        const int at = ((length[row] + places) >> shift) + k - first_page[row];
        a.page_table[(int64_t)row * a.max_pages + at] = a.free_pages[n_free - 1 - k];
      }
    }
    const int tok = begin + 4 * t;
    if (tok < a.max_tokens) {
      int pos[4], slot[4];
      int row = ok ? seq_of(first_token, a.n_rows, min(tok, max(all_tokens - 1, 0))) : 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        pos[i] = slot[i] = -1;
        if (ok && tok + i < all_tokens) {
          while (first_token[row + 1] <= tok + i) ++row;
          pos[i] = length[row] + tok + i - first_token[row];
          const int at = pos[i] >> shift, held = (length[row] + places) >> shift;
          const int p = at < held ? a.page_table[(int64_t)row * a.max_pages + at]
                                  : a.free_pages[n_free - 1 - (first_page[row] + at - held)];
          slot[i] = (p << shift) + (pos[i] & places);
        }
      }
      if (tok + 4 <= a.max_tokens) {
        *reinterpret_cast<int4*>(a.positions + tok) = make_int4(pos[0], pos[1], pos[2], pos[3]);
        *reinterpret_cast<int4*>(a.slots + tok) = make_int4(slot[0], slot[1], slot[2], slot[3]);
      } else {
        for (int i = 0; i < 4 && tok + i < a.max_tokens; ++i) {
          a.positions[tok + i] = pos[i];
          a.slots[tok + i] = slot[i];
        }
      }
    }
  }
  // After every read of the lengths and n_free (above, before a barrier): the
  // outputs may be the inputs.
  if (state && blockIdx.x == 0) {
#pragma unroll
    for (int i = 0; i < kMaxRows / kPageThreads; ++i) {
      const int row = row0 + i;
      if (i < per && row < a.n_rows) {
        a.seq_lens_out[row] = length[row] + (ok ? add[i] : 0);
        a.cu_tokens[row] = ok ? first_token[row] : 0;
      }
    }
    if (t == 0) {
      a.cu_tokens[a.n_rows] = ok ? all_tokens : 0;
      *a.n_free_out = ok ? n_free - all_pages : n_free;
      *a.status = status;
    }
  }
}

hipError_t launch_pages_extend(const PagesArgs& a, hipStream_t s) {
  const int groups = (a.max_tokens + kFillTokens - 1) / kFillTokens;
  // Workgroups start at different times: with several, the state is written
  // over the inputs by a launch of its own.
  const bool in_place = a.seq_lens_out == a.seq_lens || a.n_free_out == a.n_free;
  const bool split = groups > 1 && in_place;
  hipLaunchKernelGGL(pages_extend_kernel, dim3(groups), dim3(kPageThreads), 0, s, a, true, !split);
  if (split) hipLaunchKernelGGL(pages_extend_kernel, dim3(1), dim3(kPageThreads), 0, s, a, false, true);
  return hipGetLastError();
}

// One workgroup: sums of the released rows' pages, then their copies to the
// stack.  A row's entries are copied side by side by all threads.
__global__ __launch_bounds__(kPageThreads) void pages_release_kernel(int n_rows, int max_pages, int n_pages,
                                                                     int page_shift,
                                                                     const int32_t* __restrict__ page_table,
                                                                     int32_t* __restrict__ free_pages,
                                                                     const int32_t* __restrict__ released,
                                                                     int32_t* __restrict__ seq_lens,
                                                                     int32_t* __restrict__ n_free_io,
                                                                     int32_t* __restrict__ status_out) {
  __shared__ int sums[2 * kPageThreads / 64];
  __shared__ int first_page[kMaxRows + 1];
  const int t = threadIdx.x, places = (1 << page_shift) - 1;
  const int per = (n_rows + kPageThreads - 1) / kPageThreads;
  const int row0 = t * per;
  const int n_free = *n_free_io;
  int held[kMaxRows / kPageThreads];
  bool drop[kMaxRows / kPageThreads];
  int pages = 0;
  bool too_long = false;
#pragma unroll
  for (int i = 0; i < kMaxRows / kPageThreads; ++i) {
    held[i] = 0;
    drop[i] = false;
    const int row = row0 + i;
    if (i < per && row < n_rows) {
      const int len = seq_lens[row];
      if (len >= 0 && released[row] != 0) {
        drop[i] = true;
        held[i] = (int)(((int64_t)len + places) >> page_shift);
        too_long |= held[i] > max_pages;
      }
    }
    pages = capped_add(pages, held[i]);
  }
  int page, all_pages, none, none_all;
  scan_pair(pages, 0, sums, page, none, all_pages, none_all);
#pragma unroll
  for (int i = 0; i < kMaxRows / kPageThreads; ++i) {
    const int row = row0 + i;
    if (i < per && row < n_rows) {
      first_page[row] = page;
      page = capped_add(page, held[i]);
    }
  }
  const int status = (__syncthreads_or(too_long) ? RBS_PAGES_ROW : 0) |
                     (n_free < 0 || n_free > n_pages || all_pages > n_pages - max(n_free, 0) ? RBS_PAGES_STACK : 0);
  if (t == 0) *status_out = status;
  if (status != 0) return;
  for (int k = t; k < all_pages; k += kPageThreads) {
    const int row = seq_of(first_page, n_rows, k);
    free_pages[n_free + k] = page_table[(int64_t)row * max_pages + k - first_page[row]];
  }
#pragma unroll
  for (int i = 0; i < kMaxRows / kPageThreads; ++i)
    if (drop[i]) seq_lens[row0 + i] = -1;
  if (t == 0) *n_free_io = n_free + all_pages;
}

hipError_t launch_pages_release(int n_rows, int max_pages, int n_pages, int page_shift, const int32_t* page_table,
                                int32_t* free_pages, const int32_t* released, int32_t* seq_lens, int32_t* n_free,
                                int32_t* status, hipStream_t s) {
  hipLaunchKernelGGL(pages_release_kernel, dim3(1), dim3(kPageThreads), 0, s, n_rows, max_pages, n_pages, page_shift,
                     page_table, free_pages, released, seq_lens, n_free, status);
  return hipGetLastError();
}

// ------------------------------------------------------------------ norm, rotation, cache

// One wave works on one token's head rows, four at a time: 16 lanes to a row of
// 128, eight elements to a lane.  Lane i of a row holds pairs 4 i .. 4 i + 3, so
// that a rotation needs no other lane: elements 8 i .. 8 i + 7 where neighbours
// pair up, and 4 i .. 4 i + 3 with 4 i + rot_dim / 2 .. + 3 where halves do (past
// the rotated part, two runs of four of the rest).  The row's mean square takes
// four steps over its 16 lanes.
//
// Angles: position * inv_freq / (2 pi) in 64 bits, of which the fraction of a
// turn goes to 32-bit sine and cosine: in 32 bits alone the product would be off
// by 2^-24 of the angle itself, 0.008 of a radian at position 131072.  A wave
// computes the token's rot_dim / 2 pairs once, a pair a lane, and hands them
// round through LDS.
//
// Reads each row once and writes it once; bound by memory for prompts and by
// latency for a few tokens.
constexpr int kRopeThreads = 256;
constexpr int kRopeWaves = kRopeThreads / 64;

__device__ __forceinline__ float row_sum16(float x) {
  x += dpp_f<0xb1>(x);   // quad_perm [1, 0, 3, 2]
  x += dpp_f<0x4e>(x);   // quad_perm [2, 3, 0, 1]
  x += dpp_f<0x124>(x);  // row_ror 4
  x += dpp_f<0x128>(x);  // row_ror 8
  return x;
}

// Two fp32 to bf16 (nearest even) in one word.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((__vector_size__(2 * sizeof(__bf16))));
  const bf16x2 v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, v);
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

template <bool kInterleaved>
__global__ __launch_bounds__(kRopeThreads) void qk_norm_rope_kernel(RopeArgs a, int parts, int rows_per_part) {
  __shared__ float2 turn[kRopeWaves][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t item = (int64_t)blockIdx.x * kRopeWaves + wave;
  const int64_t tok = item / parts;
  const int part = (int)(item - tok * parts);
  const int position = tok < a.n_tokens ? a.positions[tok] : -1;
  if (position >= 0 && lane < a.rot_dim / 2) {
    const double turns = (double)position * (double)a.inv_freq[lane] * 0.15915494309189533577;
    const float part_turn = (float)(turns - rint(turns));
    float sn, cs;
    sincospif(2.f * part_turn, &sn, &cs);
    turn[wave][lane] = make_float2(cs * a.factor, sn * a.factor);
  }
  __syncthreads();
  if (position < 0) return;

  const int sub = lane >> 4, i = lane & 15;
  const int half = a.rot_dim >> 1;
  const bool rotated = 4 * i < half;
  // The lane's two runs of four elements.
  const int lo = kInterleaved ? 8 * i : rotated ? 4 * i : half + 4 * i;
  const int hi = kInterleaved ? 8 * i + 4 : rotated ? 4 * i + half : 64 + 4 * i;
  float cs[4], sn[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 v = rotated ? turn[wave][4 * i + e] : make_float2(1.f, 0.f);
    cs[e] = v.x;
    sn[e] = v.y;
  }
  float wq[8], wk[8];
  {
    auto weights = [&](const uint16_t* w, float* out) __attribute__((always_inline)) {
      const uint2 u = w == nullptr ? make_uint2(0x3f803f80u, 0x3f803f80u) : *reinterpret_cast<const uint2*>(w + lo);
      const uint2 v = w == nullptr ? make_uint2(0x3f803f80u, 0x3f803f80u) : *reinterpret_cast<const uint2*>(w + hi);
      unpack8(make_uint4(u.x, u.y, v.x, v.y), out);
    };
    weights(a.q_weight, wq);
    weights(a.k_weight, wk);
  }
  const int64_t slots = (int64_t)a.cache.n_pages << a.cache.page_shift;
  const int slot = a.cached ? a.slots[tok] : -1;
  const bool cached = slot >= 0 && slot < slots;
  const int64_t place = cached ? (int64_t)(slot >> a.cache.page_shift) * a.cache.page +
                                     (int64_t)(slot & ((1 << a.cache.page_shift) - 1)) * a.cache.tok
                               : 0;
  const int rows = a.n_q_heads + a.n_kv_heads * (a.cached ? 2 : 1);
  const int end = min(rows, (part + 1) * rows_per_part);
  for (int row = part * rows_per_part + sub; row < end; row += 4) {
    const bool is_q = row < a.n_q_heads;
    const bool is_v = row >= a.n_q_heads + a.n_kv_heads;
    const int head = is_q ? row : is_v ? row - a.n_q_heads - a.n_kv_heads : row - a.n_q_heads;
    const uint16_t* src = is_q ? a.Q + head * a.in.q_head + tok * a.in.q_tok
                               : (is_v ? a.V : a.K) + head * a.in.kv_head + tok * a.in.kv_tok;
    const uint2 u = *reinterpret_cast<const uint2*>(src + lo);
    const uint2 v = *reinterpret_cast<const uint2*>(src + hi);
    float x[8];
    unpack8(make_uint4(u.x, u.y, v.x, v.y), x);
    if (!is_v) {
      float sq = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) sq = fmaf(x[e], x[e], sq);
      sq = row_sum16(sq);  // (16 lanes of one row: all of them are here)
      const bool normed = (is_q ? a.q_weight : a.k_weight) != nullptr;
      const float inv = normed ? 1.f / sqrtf(sq * (1.f / kHeadDim) + a.eps) : 1.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] *= inv * (is_q ? wq[e] : wk[e]);
      float y[8];
      if (rotated) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int p = kInterleaved ? 2 * e : e, q = kInterleaved ? 2 * e + 1 : e + 4;
          y[p] = x[p] * cs[e] - x[q] * sn[e];
          y[q] = x[q] * cs[e] + x[p] * sn[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = y[e];
      }
    }
    const uint2 b_lo = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
    const uint2 b_hi = make_uint2(pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
    uint16_t* dst = is_q ? a.Q_out + head * a.out.q_head + tok * a.out.q_tok
                         : is_v || a.K_out == nullptr ? nullptr : a.K_out + head * a.out.kv_head + tok * a.out.kv_tok;
    if (dst != nullptr) {
      *reinterpret_cast<uint2*>(dst + lo) = b_lo;
      *reinterpret_cast<uint2*>(dst + hi) = b_hi;
    }
    if (!is_q && cached) {
      const int64_t at = place + head * a.cache.head;
      void* base = is_v ? a.cache.V : a.cache.K;
      if (a.cache.amax == nullptr) {
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(base) + at + lo) = b_lo;
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(base) + at + hi) = b_hi;
      } else {
        const float m = a.cache.amax[is_v ? a.n_kv_heads + head : head];
        const float scale = m > 0.f ? 448.f / m : 1.f;
        *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(base) + at + lo) = pack_e4m3(x, scale);
        *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(base) + at + hi) = pack_e4m3(x + 4, scale);
      }
    }
  }
}

hipError_t launch_qk_norm_rope(const RopeArgs& a, hipStream_t s) {
  const int rows = a.n_q_heads + a.n_kv_heads * (a.cached ? 2 : 1);
  int parts = 1;
  while (parts * 4 < rows && (int64_t)a.n_tokens * parts < 4096) parts *= 2;
  const int rows_per_part = ((rows + parts - 1) / parts + 3) / 4 * 4;
  const int64_t waves = (int64_t)a.n_tokens * parts;
  const dim3 grid((unsigned)((waves + kRopeWaves - 1) / kRopeWaves));
  if (a.interleaved)
    hipLaunchKernelGGL(qk_norm_rope_kernel<true>, grid, dim3(kRopeThreads), 0, s, a, parts, rows_per_part);
  else
    hipLaunchKernelGGL(qk_norm_rope_kernel<false>, grid, dim3(kRopeThreads), 0, s, a, parts, rows_per_part);
  return hipGetLastError();
}

}  // namespace rbs
