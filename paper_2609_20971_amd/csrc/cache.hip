// Rows between bf16 tensors and a paged cache of any type: keys and values
// quantised as they are written, and read back.
//
// Quantising is exact arithmetic but for its one rounding: FP8 as in the norm and
// rotation call, FP4 over a power of two for each 32 elements (fp4_scale).  16 lanes
// take a row of 128 elements, eight each; the four lanes of a quad hold a block of 32
// and agree on its scale by two exchanges.
//
// Bound by memory: each row is read once and written once.  A workgroup has 64 tokens,
// a wave 16 of them, and goes through the heads of both tensors: four rows to a load, of four tokens
// that follow each other, so that the cache's side of it is whole lines where their
// slots follow each other.
#include "paged.hpp"

namespace rbs {

namespace {

constexpr int kThreads = 256;
constexpr int kTokens = 64;            // of a workgroup
constexpr int kSteps = kTokens / 16;   // loads in flight: four rows of each of the four waves
// Workgroups that a call of few tokens is spread over, by heads.  131072 FP4 tokens of 4
// heads are written in 68 us at 2048, 70.5 at 4096 and 78 at 16384 (a wave's next head is
// the next line of the same page); 32 rows of 100 to 9000 tokens, 8 heads, are read in
// 78, 73 and 75 us (call after call, three sets of rows in turn).
constexpr int kWriteSpread = 2048, kReadSpread = 4096;

// A call that moves this many bytes or more loads past the caches, which its loads would
// only empty, and stores through them.  After a copy of 1 GB the same rows are read in
// 70 us for FP4, 68 for FP8 and 103 for BF16; in 83, 90 and 115 with stores past the
// caches too, in 88, 101 and 142 with the stores alone.  131072 tokens of 4 heads are
// written in 71 us (FP4), 75 (FP8) and 88 (BF16): 4.8, 5.4 and 6.1 TB/s; FP4 and BF16 in 72 and 109
// with stores past the caches too.
constexpr int64_t kCachedBytes = int64_t(64) << 20;

template <int kFmt>
constexpr int kCodeBytes = kFmt == kCacheFp4 ? kHeadDim / 2 : kFmt == kCacheFp8 ? kHeadDim : 2 * kHeadDim;

// The lanes' largest magnitude over each quad.
__device__ __forceinline__ uint32_t quad_top(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xb1, 0xf, 0xf, false));
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4e, 0xf, 0xf, false));
}

// Element offset of a slot in the cache (-1: none).
__device__ __forceinline__ int64_t place_of(const CacheView& c, int64_t slot) {
  if (slot < 0 || slot >= (int64_t)c.n_pages << c.page_shift) return -1;
  return (slot >> c.page_shift) * c.page + (slot & ((1 << c.page_shift) - 1)) * c.tok;
}

// The share of the heads of both tensors (K's, then V's) of this workgroup.
__device__ __forceinline__ void my_rows(const MoveArgs& a, int parts, int* from, int* to) {
  const int part = blockIdx.x % parts, rows = 2 * a.n_kv_heads;
  *from = rows * part / parts;
  *to = rows * (part + 1) / parts;
}

template <int kFmt, bool kOnce>
__global__ __launch_bounds__(kThreads) void cache_write_kernel(MoveArgs a, int parts) {
  const int sub = threadIdx.x >> 4, i = threadIdx.x & 15;
  const int64_t tok0 = (int64_t)(blockIdx.x / parts) * kTokens;
  int64_t place[kSteps];
#pragma unroll
  for (int u = 0; u < kSteps; ++u) {
    const int64_t t = tok0 + 16 * u + sub;
    place[u] = t < a.n_tokens ? place_of(a.cache, a.slots[t]) : -1;
  }
  int from, to;
  my_rows(a, parts, &from, &to);
  for (int row = from; row < to; ++row) {
    const bool is_v = row >= a.n_kv_heads;
    const int h = is_v ? row - a.n_kv_heads : row;
    const uint16_t* src = is_v ? a.V + h * a.v_head : a.K + h * a.k_head;
    const int64_t tok = is_v ? a.v_tok : a.k_tok;
    uint32_t w[kSteps][4];
#pragma unroll
    for (int u = 0; u < kSteps; ++u)
      if (place[u] >= 0) load_words<4, kOnce>(src + (tok0 + 16 * u + sub) * tok + 8 * i, w[u]);
    float scale = 1.f;
    if (kFmt == kCacheFp8) {
      const float m = a.cache.amax[row];
      scale = m > 0.f ? 448.f / m : 1.f;
    }
    char* codes = static_cast<char*>(is_v ? a.cache.V : a.cache.K);
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
      if (place[u] < 0) continue;  // (the row's 16 lanes together)
      const int64_t at = place[u] + h * a.cache.head;
      char* out = codes + at * kCodeBytes<kFmt> / kHeadDim + i * (kCodeBytes<kFmt> / 16);
      if (kFmt == kCacheBf16) {
        store_words<4, false>(out, w[u]);
      } else if (kFmt == kCacheFp8) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[2 * e] = bf16_lo(w[u][e]);
          x[2 * e + 1] = bf16_hi(w[u][e]);
        }
        const uint32_t c[2] = {pack_e4m3(x, scale), pack_e4m3(x + 4, scale)};
        store_words<2, false>(out, c);
      } else {
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) top = max(top, max(w[u][e] & 0x7fffu, (w[u][e] >> 16) & 0x7fffu));
        const uint32_t s = fp4_scale(quad_top(top));
        const uint32_t c[1] = {pack_e2m1(w[u], s)};
        store_words<1, false>(out, c);
        if ((i & 3) == 0) static_cast<uint8_t*>(is_v ? a.cache.V_scale : a.cache.K_scale)[at / 32 + (i >> 2)] = (uint8_t)s;
      }
    }
  }
}

// The rows' offsets go to LDS, where each token finds its row.
template <int kFmt, bool kOnce>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(MoveArgs a, int parts) {
  __shared__ int first[kMaxRows + 1];
  __shared__ int64_t places[kTokens];
  const int64_t tok0 = (int64_t)(blockIdx.x / parts) * kTokens;
  for (int r = threadIdx.x; r <= a.n_rows; r += kThreads) first[r] = a.cu_tokens[r];
  __syncthreads();
  if (threadIdx.x < kTokens) {
    const int64_t t = tok0 + threadIdx.x;
    int64_t place = -1;
    if (t < a.n_tokens) {
      const int row = seq_of(first, a.n_rows, (int)t);
      if (t >= first[row] && t < first[row + 1]) {
        const int64_t p = (a.starts == nullptr ? 0 : (int64_t)a.starts[row]) + t - first[row];
        if (p >= 0 && p < (int64_t)a.max_pages << a.cache.page_shift) {
          const int page = a.page_table[(int64_t)row * a.max_pages + (p >> a.cache.page_shift)];
          place = (int64_t)min(max(page, 0), a.cache.n_pages - 1) * a.cache.page +
                  (p & ((1 << a.cache.page_shift) - 1)) * a.cache.tok;
        }
      }
    }
    places[threadIdx.x] = place;
  }
  __syncthreads();
  const int sub = threadIdx.x >> 4, i = threadIdx.x & 15;
  int64_t place[kSteps];
#pragma unroll
  for (int u = 0; u < kSteps; ++u) place[u] = places[16 * u + sub];
  int from, to;
  my_rows(a, parts, &from, &to);
  for (int row = from; row < to; ++row) {
    const bool is_v = row >= a.n_kv_heads;
    const int h = is_v ? row - a.n_kv_heads : row;
    const char* codes = static_cast<const char*>(is_v ? a.cache.V : a.cache.K);
    const uint8_t* scales = static_cast<const uint8_t*>(is_v ? a.cache.V_scale : a.cache.K_scale);
    constexpr int kWords = kCodeBytes<kFmt> / 64;
    uint32_t w[kSteps][kWords], s[kSteps] = {};
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
      if (place[u] < 0) continue;
      const int64_t at = place[u] + h * a.cache.head;
      load_words<kWords, kOnce>(codes + at * kCodeBytes<kFmt> / kHeadDim + i * (kCodeBytes<kFmt> / 16), w[u]);
      if (kFmt == kCacheFp4) s[u] = scales[at / 32 + (i >> 2)];
    }
    float scale = 1.f;
    if (kFmt == kCacheFp8) {
      const float m = a.cache.amax[row];
      scale = m > 0.f ? m / 448.f : 1.f;
    }
    uint16_t* dst = is_v ? a.V + h * a.v_head : a.K + h * a.k_head;
    const int64_t tok = is_v ? a.v_tok : a.k_tok;
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
      if (place[u] < 0) continue;
      uint32_t out[4];
      if constexpr (kFmt == kCacheBf16) {
#pragma unroll
        for (int e = 0; e < 4; ++e) out[e] = w[u][e];
      } else if constexpr (kFmt == kCacheFp8) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int c = (int)w[u][e];
          out[2 * e] = two_bf16(__builtin_amdgcn_cvt_f32_fp8(c, 0) * scale, __builtin_amdgcn_cvt_f32_fp8(c, 1) * scale);
          out[2 * e + 1] = two_bf16(__builtin_amdgcn_cvt_f32_fp8(c, 2) * scale, __builtin_amdgcn_cvt_f32_fp8(c, 3) * scale);
        }
      } else {
        const uint4 v = widen_e2m1(w[u][0], s[u] << 23);
        out[0] = v.x; out[1] = v.y; out[2] = v.z; out[3] = v.w;
      }
      store_words<4, false>(dst + (tok0 + 16 * u + sub) * tok + 8 * i, out);
    }
  }
}

// Workgroups and the parts of their heads; whether its loads go past the caches.
void launch_of(const MoveArgs& a, int code_bytes, int spread, int* groups, int* parts, bool* once) {
  const int64_t chunks = ((int64_t)a.n_tokens + kTokens - 1) / kTokens;
  *parts = 1;
  while (*parts < 2 * a.n_kv_heads && chunks * *parts < spread) ++*parts;
  *groups = (int)(chunks * *parts);
  *once = (int64_t)a.n_tokens * 2 * a.n_kv_heads * (2 * kHeadDim + code_bytes) >= kCachedBytes;
}

template <int kFmt>
hipError_t launch_write(const MoveArgs& a, hipStream_t s) {
  int groups, parts;
  bool once;
  launch_of(a, kCodeBytes<kFmt>, kWriteSpread, &groups, &parts, &once);
  const auto kernel = once ? cache_write_kernel<kFmt, true> : cache_write_kernel<kFmt, false>;
  hipLaunchKernelGGL(kernel, dim3(groups), dim3(kThreads), 0, s, a, parts);
  return hipGetLastError();
}

template <int kFmt>
hipError_t launch_read(const MoveArgs& a, hipStream_t s) {
  int groups, parts;
  bool once;
  launch_of(a, kCodeBytes<kFmt>, kReadSpread, &groups, &parts, &once);
  const auto kernel = once ? cache_read_kernel<kFmt, true> : cache_read_kernel<kFmt, false>;
  hipLaunchKernelGGL(kernel, dim3(groups), dim3(kThreads), 0, s, a, parts);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_write(const MoveArgs& a, hipStream_t s) {
  switch (a.cache.format) {
    case kCacheBf16: return launch_write<kCacheBf16>(a, s);
    case kCacheFp8: return launch_write<kCacheFp8>(a, s);
    case kCacheFp4: return launch_write<kCacheFp4>(a, s);
    default: return hipErrorInvalidValue;
  }
}

hipError_t launch_cache_read(const MoveArgs& a, hipStream_t s) {
  switch (a.cache.format) {
    case kCacheBf16: return launch_read<kCacheBf16>(a, s);
    case kCacheFp8: return launch_read<kCacheFp8>(a, s);
    case kCacheFp4: return launch_read<kCacheFp4>(a, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace rbs
