// Attention of one new token per row over a paged key-value cache.
#include "rbs_device.hpp"
#include "rbs_launch.hpp"

namespace rbs {

size_t decode_workspace_bytes() { return 16; }

// E4M3 code -> fp32, through the hardware conversion of one byte of a word.
template <int kByte>
__device__ __forceinline__ float e4m3(uint32_t w) {
  return __builtin_amdgcn_cvt_f32_fp8((int)w, kByte);
}

// One workgroup per (row, query head).  16 lanes hold a key's 128 elements,
// eight each; a wave takes four keys at a time and the workgroup 16, each group
// of 16 lanes with a softmax state (running maximum, sum, weighted values) of its
// own, joined at the end.
template <bool kFp8>
__global__ __launch_bounds__(256) void paged_decode_kernel(DecodeArgs a) {
  const int row = blockIdx.x, h = blockIdx.y, g = h / (a.n_q_heads / a.n_kv_heads);
  const int lane = threadIdx.x & 63, i = lane & 15, group = threadIdx.x >> 4;
  const int shift = a.cache.page_shift;
  int len = a.seq_lens[row];
  if (len < 0) return;
  len = min((int64_t)len, (int64_t)a.max_pages << shift);
  const int32_t* table = a.page_table + (int64_t)row * a.max_pages;
  float q[8];
  unpack8(*reinterpret_cast<const uint4*>(a.Q + h * a.q_head + row * a.q_tok + 8 * i), q);
  const float k_scale = kFp8 && a.cache.amax[g] > 0.f ? a.cache.amax[g] / 448.f : 1.f;
  const float v_scale = kFp8 && a.cache.amax[a.n_kv_heads + g] > 0.f ? a.cache.amax[a.n_kv_heads + g] / 448.f : 1.f;
  auto load = [&](const void* base, int64_t at, float* out) __attribute__((always_inline)) {
    if (kFp8) {
      const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(base) + at);
      out[0] = e4m3<0>(w.x); out[1] = e4m3<1>(w.x); out[2] = e4m3<2>(w.x); out[3] = e4m3<3>(w.x);
      out[4] = e4m3<0>(w.y); out[5] = e4m3<1>(w.y); out[6] = e4m3<2>(w.y); out[7] = e4m3<3>(w.y);
    } else {
      unpack8(*reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(base) + at), out);
    }
  };
  float m = -INFINITY, l = 0.f, o[8] = {};
  for (int j = group; j < len; j += 16) {
    const int page = min(max(table[j >> shift], 0), a.cache.n_pages - 1);
    const int64_t at = page * a.cache.page + g * a.cache.head + (int64_t)(j & ((1 << shift) - 1)) * a.cache.tok + 8 * i;
    float k[8], v[8], x = 0.f;
    load(a.cache.K, at, k);
    load(a.cache.V, at, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) x = fmaf(q[e], k[e], x);
    x += dpp_f<0xb1>(x);
    x += dpp_f<0x4e>(x);
    x += dpp_f<0x124>(x);
    x += dpp_f<0x128>(x);
    x *= k_scale * a.scale;
    const float top = fmaxf(m, x), keep = m == top ? 1.f : expf(m - top), p = x == top ? 1.f : expf(x - top);
    m = top;
    l = l * keep + p;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = o[e] * keep + p * v[e];
  }
  __shared__ float ms[16], ls[16], os[16][kHeadDim];
  if (i == 0) {
    ms[group] = m;
    ls[group] = l;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) os[group][8 * i + e] = o[e];
  __syncthreads();
  if (threadIdx.x >= kHeadDim) return;
  const int e = threadIdx.x;
  float top = -INFINITY, sum = 0.f, out = 0.f;
  for (int w = 0; w < 16; ++w)
    if (ls[w] > 0.f) top = fmaxf(top, ms[w]);
  for (int w = 0; w < 16; ++w) {
    if (ls[w] == 0.f) continue;  // no key here
    const float f = ms[w] == top ? 1.f : expf(ms[w] - top);
    sum += ls[w] * f;
    out += os[w][e] * f;
  }
  out = len > 0 ? out * v_scale / sum : 0.f;
  const __bf16 b = (__bf16)out;
  a.O[h * a.q_head + row * a.q_tok + e] = __builtin_bit_cast(uint16_t, b);
  if (e == 0 && a.lse != nullptr) a.lse[(int64_t)h * a.n_rows + row] = len > 0 ? top + logf(sum) : -INFINITY;
}

hipError_t launch_paged_decode(const DecodeArgs& a, hipStream_t s) {
  const dim3 grid(a.n_rows, a.n_q_heads);
  if (a.cache.amax != nullptr)
    hipLaunchKernelGGL(paged_decode_kernel<true>, grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(paged_decode_kernel<false>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace rbs
