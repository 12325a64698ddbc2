// Around a paged key-value cache: pages and slots of a batch's new tokens, pages
// given back, and queries and keys normed, rotated and put into the cache.
#include "../../include/rbs.h"
#include "paged.hpp"

namespace rbs {

// ------------------------------------------------------------------ pages

constexpr int kPageThreads = 256;
constexpr int kRowsPerThread = kMaxRows / kPageThreads;
constexpr int kFillTokens = 4 * kPageThreads;  // tokens (and new pages) of one workgroup
constexpr int kMost = 1 << 29;                 // sums stop here, past every limit that they are compared with

__device__ __forceinline__ int capped_add(int a, int b) { return min(a + b, kMost); }  // a, b in 0 .. kMost

// Sums of two counts over the threads before this one, and over all of them.
// Capped addition of nonnegative numbers is associative, so that the order of
// the partial sums does not matter.
__device__ __forceinline__ void scan_pair(int a, int b, int* sums, int& a_before, int& b_before, int& a_all,
                                          int& b_all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int x = wave_scan(a, capped_add), y = wave_scan(b, capped_add);
  constexpr int kWaves = kPageThreads / 64;
  if (lane == 63) {
    sums[wave] = x;
    sums[kWaves + wave] = y;
  }
  __syncthreads();
  a_before = __builtin_amdgcn_update_dpp(0, x, 0x138, 0xf, 0xf, false);  // wave_shr 1
  b_before = __builtin_amdgcn_update_dpp(0, y, 0x138, 0xf, 0xf, false);
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
//
// kOne: a token each (a decode step).  A row's thread then writes the row's token
// itself, and asks for its last page before the sums (48 rows 6.3 -> 2.8 us).
template <bool kOne>
__global__ __launch_bounds__(kPageThreads) void pages_extend_kernel(PagesArgs a, bool fill, bool state) {
  __shared__ int sums[2 * kPageThreads / 64];
  __shared__ int first_token[kMaxRows + 1], first_page[kMaxRows + 1], length[kMaxRows];
  const int t = threadIdx.x, shift = a.page_shift, places = (1 << shift) - 1;
  const int per = (a.n_rows + kPageThreads - 1) / kPageThreads;  // rows per thread
  const int row0 = t * per;
  const int n_free = *a.n_free;
  int add[kRowsPerThread], need[kRowsPerThread], page_of[kOne ? kRowsPerThread : 1];
  int tokens = 0, pages = 0;
  bool too_long = false;
  // This workgroup's share of the new pages, before it is known how many there are.
  constexpr int kTaken = kOne ? 1 : kFillTokens / kPageThreads;
  int taken[kTaken];
  if (!kOne) {
#pragma unroll
    for (int i = 0; i < kTaken; ++i) {
      const int k = (int)blockIdx.x * kFillTokens + i * kPageThreads + t;
      taken[i] = a.free_pages[max(min(max(n_free, 0), a.n_pages) - 1 - k, 0)];
    }
  }
#pragma unroll
  for (int i = 0; i < kRowsPerThread; ++i) add[i] = need[i] = 0;
#pragma unroll
  for (int i = 0; i < kRowsPerThread; ++i) {
    const int row = row0 + i;
    if (i >= per) break;
    if (row < a.n_rows) {
      const int len = a.seq_lens[row], more = kOne ? 1 : max(a.new_tokens[row], 0);
      length[row] = len;
      if (len >= 0) {
        if (kOne) page_of[i] = a.page_table[(int64_t)row * a.max_pages + min(len >> shift, a.max_pages - 1)];
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
  for (int i = 0; i < kRowsPerThread; ++i) {
    const int row = row0 + i;
    if (i >= per) break;
    if (row < a.n_rows) {
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
  const int status = (all_pages > max(n_free, 0) ? RBS_PAGES_FEW : 0) |
                     (__syncthreads_or(too_long) ? RBS_PAGES_ROW : 0) |
                     (all_tokens > a.max_tokens ? RBS_PAGES_TOKENS : 0) |
                     (n_free < 0 || n_free > a.n_pages ? RBS_PAGES_STACK : 0);
  const bool ok = status == 0;

  if (fill) {
    const int begin = blockIdx.x * kFillTokens;
    if (kOne) {
      if (blockIdx.x == 0 && ok) {
#pragma unroll
        for (int i = 0; i < kRowsPerThread; ++i) {
          const int row = row0 + i;
          if (i >= per) break;
          if (row >= a.n_rows || add[i] == 0) continue;
          const int len = length[row], tok = first_token[row];
          if (need[i] != 0) {  // (its length is a whole number of pages)
            page_of[i] = a.free_pages[n_free - 1 - first_page[row]];
            a.page_table[(int64_t)row * a.max_pages + (len >> shift)] = page_of[i];
          }
          a.positions[tok] = len;
          a.slots[tok] = (page_of[i] << shift) + (len & places);
        }
      }
      for (int tok = max(begin, ok ? all_tokens : 0) + t; tok < min(begin + kFillTokens, a.max_tokens);
           tok += kPageThreads)
        a.positions[tok] = a.slots[tok] = -1;
    } else {
      // Four tokens a thread: where each one's page number stands, then all four loads
      // at once (tokens with none read the stack's first entry, for nothing).
      const int tok = begin + 4 * t;
      int pos[4];
      const int32_t* page_at[4];
      int row = ok ? seq_of(first_token, a.n_rows, min(tok, max(all_tokens - 1, 0))) : 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        pos[i] = -1;
        page_at[i] = a.free_pages;
        if (ok && tok + i < all_tokens) {
          if (first_token[row + 1] <= tok + i && first_token[++row + 1] <= tok + i)
            row = seq_of(first_token, a.n_rows, tok + i);  // (many rows may take none)
          pos[i] = length[row] + tok + i - first_token[row];
          const int at = pos[i] >> shift, held = (length[row] + places) >> shift;
          page_at[i] = at < held ? a.page_table + (int64_t)row * a.max_pages + at
                                 : a.free_pages + (n_free - 1 - (first_page[row] + at - held));
        }
      }
      int slot[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) slot[i] = *page_at[i];
#pragma unroll
      for (int i = 0; i < 4; ++i) slot[i] = pos[i] < 0 ? -1 : (slot[i] << shift) + (pos[i] & places);
      if (tok + 4 <= a.max_tokens) {
        *reinterpret_cast<int4*>(a.positions + tok) = make_int4(pos[0], pos[1], pos[2], pos[3]);
        *reinterpret_cast<int4*>(a.slots + tok) = make_int4(slot[0], slot[1], slot[2], slot[3]);
      } else {
        for (int i = 0; i < 4 && tok + i < a.max_tokens; ++i) {
          a.positions[tok + i] = pos[i];
          a.slots[tok + i] = slot[i];
        }
      }
      if (ok) {
#pragma unroll
        for (int i = 0; i < kTaken; ++i) {
          const int k = begin + i * kPageThreads + t;
          if (k >= all_pages) break;
          const int row = seq_of(first_page, a.n_rows, k);
          const int at = ((length[row] + places) >> shift) + k - first_page[row];
          a.page_table[(int64_t)row * a.max_pages + at] = taken[i];
        }
      }
    }
  }
  // After every read of the lengths and n_free (above, before a barrier): the
  // outputs may be the inputs.
  if (state && blockIdx.x == 0) {
#pragma unroll
    for (int i = 0; i < kRowsPerThread; ++i) {
      const int row = row0 + i;
      if (i >= per) break;
      if (row < a.n_rows) {
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
  const auto kernel = a.new_tokens == nullptr ? pages_extend_kernel<true> : pages_extend_kernel<false>;
  hipLaunchKernelGGL(kernel, dim3(groups), dim3(kPageThreads), 0, s, a, true, !split);
  if (split) hipLaunchKernelGGL(kernel, dim3(1), dim3(kPageThreads), 0, s, a, false, true);
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
  int held[kRowsPerThread];
  bool drop[kRowsPerThread];
  int pages = 0;
  bool too_long = false;
#pragma unroll
  for (int i = 0; i < kRowsPerThread; ++i) {
    held[i] = 0;
    drop[i] = false;
  }
#pragma unroll
  for (int i = 0; i < kRowsPerThread; ++i) {
    const int row = row0 + i;
    if (i >= per) break;
    if (row < n_rows) {
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
  for (int i = 0; i < kRowsPerThread; ++i) {
    const int row = row0 + i;
    if (i >= per) break;
    if (row < n_rows) {
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
  for (int i = 0; i < kRowsPerThread; ++i)
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

// A wave works on one token's head rows, 64 / kLanes of them at a time: kLanes lanes
// to a row of 128, two runs of kRun = 64 / kLanes elements to a lane.  Lane i of a
// row holds pairs kRun i .. + kRun - 1, so that a rotation needs no other lane: runs
// 2 i and 2 i + 1 where neighbours pair up, and run i and the one rot_dim / 2 after
// it where halves do (past the rotated part, two runs of the rest).  Runs of eight
// elements, 16 bytes, move a row with half as many loads as runs of four, and need
// pairs in multiples of eight.
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
// From this many bytes of rows on a call reads and writes past the caches, and in
// runs of eight: 128K tokens of 32 / 4 heads (1.3 GB) cached, in runs of four 534 us,
// past the caches 490, in runs of eight as well 478; 8000 tokens (82 MB) 34.2 and
// 33.4.  Below, the next call finds the rows in the Infinity Cache, and what runs
// of eight save is less than their fewer waves cost: 3001 tokens of 28 / 4 heads (28
// MB) 12.4 cached in runs of four, 14.9 in runs of eight, 17.0 past the caches as
// well; 96 of 64 / 8 3.9 and 4.3.  With K and V into a cache, 32 / 4 heads: 512 tokens 5.2 us
// (bf16), 6.0 (FP8, 4 bits), 8000 33 to 34, 131072 470, 452 and 437.
constexpr int64_t kRopeCachedBytes = int64_t(64) << 20;
// Waves that a call of few tokens is spread over, a token's rows in several parts.
// 2048 / 4096 / 8192: 512 tokens of 32 / 4 heads 5.2 / 4.9 / 4.9 us, 1500 10.8 / 10.1 /
// 10.4, 3001 of 28 / 4 13.4 / 12.5 / 13.1, 2000 of 8 / 1 5.1 / 5.7 / 5.7.
constexpr int kRopeSpread = 4096;

template <int kLanes>
__device__ __forceinline__ float row_sum(float x) {
  x += dpp_f<0xb1>(x);                      // quad_perm [1, 0, 3, 2]
  x += dpp_f<0x4e>(x);                      // quad_perm [2, 3, 0, 1]
  x += dpp_f<0x141>(x);                     // row_half_mirror: the other quad of eight lanes
  if (kLanes == 16) x += dpp_f<0x128>(x);   // row_ror 8
  return x;
}

// The largest of each half word over the lanes of a row, in all of them.
template <int kLanes>
__device__ __forceinline__ uint32_t row_top(uint32_t x) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  auto top = [](uint32_t a, int b) __attribute__((always_inline)) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
  };
  x = top(x, __builtin_amdgcn_update_dpp(0, (int)x, 0xb1, 0xf, 0xf, false));   // as in row_sum
  x = top(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x4e, 0xf, 0xf, false));
  x = top(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xf, 0xf, false));
  if (kLanes == 16) x = top(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xf, 0xf, false));
  return x;
}

// The largest magnitude (bits of bf16) of a run.
template <int kWords>
__device__ __forceinline__ uint32_t run_top(const uint32_t* w) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < kWords; ++e) top = max(top, max(w[e] & 0x7fffu, (w[e] >> 16) & 0x7fffu));
  return top;
}

// E2M1 codes of a run of eight elements, or of four in the low half.
template <int kWords>
__device__ __forceinline__ uint32_t pack_run(const uint32_t* w, uint32_t scale) {
  const uint32_t x[4] = {w[0], w[1], kWords == 4 ? w[kWords - 2] : 0u, kWords == 4 ? w[kWords - 1] : 0u};
  return pack_e2m1(x, scale);
}

// kFp4: into a cache in 4 bits, by code of its own, whose registers would cost the other
// formats two of eight waves (512 tokens of 32 / 4 heads into FP8 6.15 us and not 5.95, 1500 into bf16 9.6
// and not 9.4).
template <int kLanes, bool kInterleaved, bool kOnce, bool kFp4>
__global__ __launch_bounds__(kRopeThreads) void qk_norm_rope_kernel(RopeArgs a, int parts, int rows_per_part) {
  constexpr int kRun = 64 / kLanes, kRows = 64 / kLanes, kUnroll = 2;
  __shared__ __align__(16) float cosines[kRopeWaves][64], sines[kRopeWaves][64];
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
    cosines[wave][lane] = cs * a.factor;
    sines[wave][lane] = sn * a.factor;
  }
  __syncthreads();
  if (position < 0) return;

  const int sub = lane / kLanes, i = lane % kLanes;
  const int half = a.rot_dim >> 1;
  const bool rotated = kRun * i < half;
  // The lane's two runs.
  const int lo = kInterleaved ? 2 * kRun * i : rotated ? kRun * i : half + kRun * i;
  const int hi = kInterleaved ? lo + kRun : rotated ? lo + half : 64 + kRun * i;
  float cs[kRun], sn[kRun];
#pragma unroll
  for (int e = 0; e < kRun; ++e) {
    cs[e] = rotated ? cosines[wave][kRun * i + e] : 1.f;
    sn[e] = rotated ? sines[wave][kRun * i + e] : 0.f;
  }
  // (Weights of the two tensors in turn, kept as bf16 pairs.)
  uint32_t wq[kRun], wk[kRun];
  auto weights = [&](const uint16_t* w, uint32_t* out) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < kRun; ++e) out[e] = 0x3f803f80u;
    if (w == nullptr) return;
    load_words<kRun / 2, false>(w + lo, out);
    load_words<kRun / 2, false>(w + hi, out + kRun / 2);
  };
  weights(a.q_weight, wq);
  weights(a.k_weight, wk);
  const int64_t slots = (int64_t)a.cache.n_pages << a.cache.page_shift;
  const int slot = a.cached ? a.slots[tok] : -1;
  const bool cached = slot >= 0 && slot < slots;
  const int64_t place = cached ? (int64_t)(slot >> a.cache.page_shift) * a.cache.page +
                                     (int64_t)(slot & ((1 << a.cache.page_shift) - 1)) * a.cache.tok
                               : 0;
  const int rows = a.n_q_heads + a.n_kv_heads * (a.cached ? 2 : 1);
  const int end = min(rows, (part + 1) * rows_per_part);

  for (int row0 = part * rows_per_part + sub; row0 < end; row0 += kRows * kUnroll) {
    uint32_t w[kUnroll][kRun];  // lo's elements in the first half of the words, then hi's
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int row = row0 + u * kRows;
      if (row < end) {
        const bool is_q = row < a.n_q_heads, is_v = row >= a.n_q_heads + a.n_kv_heads;
        const int head = is_q ? row : is_v ? row - a.n_q_heads - a.n_kv_heads : row - a.n_q_heads;
        const uint16_t* src = is_q ? a.Q + head * a.in.q_head + tok * a.in.q_tok
                                   : (is_v ? a.V : a.K) + head * a.in.kv_head + tok * a.in.kv_tok;
        load_words<kRun / 2, kOnce>(src + lo, w[u]);
        load_words<kRun / 2, kOnce>(src + hi, w[u] + kRun / 2);
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int row = row0 + u * kRows;
      if (row >= end) break;
      const bool is_q = row < a.n_q_heads, is_v = row >= a.n_q_heads + a.n_kv_heads;
      const int head = is_q ? row : is_v ? row - a.n_q_heads - a.n_kv_heads : row - a.n_q_heads;
      float x[2 * kRun];
#pragma unroll
      for (int e = 0; e < kRun; ++e) {
        x[2 * e] = bf16_lo(w[u][e]);
        x[2 * e + 1] = bf16_hi(w[u][e]);
      }
      if (!is_v) {
        float sq = 0.f;
#pragma unroll
        for (int e = 0; e < 2 * kRun; ++e) sq = fmaf(x[e], x[e], sq);
        sq = row_sum<kLanes>(sq);  // (the row's lanes are all here)
        const bool normed = (is_q ? a.q_weight : a.k_weight) != nullptr;
        const float inv = normed ? 1.f / sqrtf(sq * (1.f / kHeadDim) + a.eps) : 1.f;
#pragma unroll
        for (int e = 0; e < kRun; ++e) {
          const uint32_t g = is_q ? wq[e] : wk[e];
          x[2 * e] *= inv * bf16_lo(g);
          x[2 * e + 1] *= inv * bf16_hi(g);
        }
        if (rotated) {
#pragma unroll
          for (int e = 0; e < kRun; ++e) {
            const int p = kInterleaved ? 2 * e : e, q = kInterleaved ? 2 * e + 1 : e + kRun;
            const float xp = x[p], xq = x[q];
            x[p] = xp * cs[e] - xq * sn[e];
            x[q] = xq * cs[e] + xp * sn[e];
          }
        }
      }
      uint32_t b[kRun];
#pragma unroll
      for (int e = 0; e < kRun; ++e) b[e] = two_bf16(x[2 * e], x[2 * e + 1]);
      if (is_v) {  // (as it came: a NaN keeps its bits)
#pragma unroll
        for (int e = 0; e < kRun; ++e) b[e] = w[u][e];
      }
      uint16_t* dst = is_q ? a.Q_out + head * a.out.q_head + tok * a.out.q_tok
                           : is_v || a.K_out == nullptr ? nullptr
                                                        : a.K_out + head * a.out.kv_head + tok * a.out.kv_tok;
      if (dst != nullptr) {
        store_words<kRun / 2, kOnce>(dst + lo, b);
        store_words<kRun / 2, kOnce>(dst + hi, b + kRun / 2);
      }
      if (!is_q && cached) {
        const int64_t at = place + head * a.cache.head;
        void* base = is_v ? a.cache.V : a.cache.K;
        if constexpr (kFp4) {
          // Of the row as it is written to K_out, in bf16.  A run lies within one
          // block of 32 elements; the four blocks' largest go round the row's lanes in
          // two words.
          constexpr int kWords = kRun / 2;
          const uint32_t lo_top = run_top<kWords>(b), hi_top = run_top<kWords>(b + kWords);
          const int lo_block = lo >> 5, hi_block = hi >> 5;
          uint32_t tops[2];
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const uint32_t even = max(lo_block == 2 * x ? lo_top : 0u, hi_block == 2 * x ? hi_top : 0u);
            const uint32_t odd = max(lo_block == 2 * x + 1 ? lo_top : 0u, hi_block == 2 * x + 1 ? hi_top : 0u);
            tops[x] = row_top<kLanes>(even | odd << 16);
          }
          uint32_t scales = 0;
#pragma unroll
          for (int x = 0; x < 4; ++x) scales |= fp4_scale((tops[x >> 1] >> (16 * (x & 1))) & 0x7fffu) << (8 * x);
          const uint32_t lo_codes = pack_run<kWords>(b, (scales >> (8 * lo_block)) & 255u);
          const uint32_t hi_codes = pack_run<kWords>(b + kWords, (scales >> (8 * hi_block)) & 255u);
          uint8_t* codes = static_cast<uint8_t*>(base) + (at >> 1);
          if (kRun == 8) {
            *reinterpret_cast<uint32_t*>(codes + (lo >> 1)) = lo_codes;
            *reinterpret_cast<uint32_t*>(codes + (hi >> 1)) = hi_codes;
          } else {
            *reinterpret_cast<uint16_t*>(codes + (lo >> 1)) = (uint16_t)lo_codes;
            *reinterpret_cast<uint16_t*>(codes + (hi >> 1)) = (uint16_t)hi_codes;
          }
          if (i == 0)
            *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(is_v ? a.cache.V_scale : a.cache.K_scale) + (at >> 5)) = scales;
        } else if (a.cache.amax == nullptr) {
          store_words<kRun / 2, kOnce>(static_cast<uint16_t*>(base) + at + lo, b);
          store_words<kRun / 2, kOnce>(static_cast<uint16_t*>(base) + at + hi, b + kRun / 2);
        } else {
          const float m = a.cache.amax[is_v ? a.n_kv_heads + head : head];
          const float scale = m > 0.f ? 448.f / m : 1.f;
          uint32_t code[kRun / 2];
#pragma unroll
          for (int e = 0; e < kRun / 2; ++e) code[e] = pack_e4m3(x + 4 * e, scale);
          store_words<kRun / 4, kOnce>(static_cast<uint8_t*>(base) + at + lo, code);
          store_words<kRun / 4, kOnce>(static_cast<uint8_t*>(base) + at + hi, code + kRun / 4);
        }
      }
    }
  }
}

hipError_t launch_qk_norm_rope(const RopeArgs& a, hipStream_t s) {
  const int rows = a.n_q_heads + a.n_kv_heads * (a.cached ? 2 : 1);
  const bool once = (int64_t)a.n_tokens * rows * (2 * kHeadDim) >= kRopeCachedBytes;
  const bool wide = once && a.rot_dim % 16 == 0;
  const int at_once = wide ? 8 : 4;
  int parts = 1;
  while (parts * at_once < rows && (int64_t)a.n_tokens * parts < kRopeSpread) parts *= 2;
  const int rows_per_part = ((rows + parts - 1) / parts + at_once - 1) / at_once * at_once;
  parts = (rows + rows_per_part - 1) / rows_per_part;
  const int64_t waves = (int64_t)a.n_tokens * parts;
  const dim3 grid((unsigned)((waves + kRopeWaves - 1) / kRopeWaves));
  using Kernel = void (*)(RopeArgs, int, int);
  static constexpr Kernel kernels[2][3][2] = {
      {{qk_norm_rope_kernel<16, false, false, false>, qk_norm_rope_kernel<16, true, false, false>},
       {qk_norm_rope_kernel<16, false, true, false>, qk_norm_rope_kernel<16, true, true, false>},
       {qk_norm_rope_kernel<8, false, true, false>, qk_norm_rope_kernel<8, true, true, false>}},
      {{qk_norm_rope_kernel<16, false, false, true>, qk_norm_rope_kernel<16, true, false, true>},
       {qk_norm_rope_kernel<16, false, true, true>, qk_norm_rope_kernel<16, true, true, true>},
       {qk_norm_rope_kernel<8, false, true, true>, qk_norm_rope_kernel<8, true, true, true>}}};
  const bool fp4 = a.cached && a.cache.format == kCacheFp4;
  hipLaunchKernelGGL(kernels[fp4][wide ? 2 : once][a.interleaved], grid, dim3(kRopeThreads), 0, s, a, parts, rows_per_part);
  return hipGetLastError();
}

}  // namespace rbs
