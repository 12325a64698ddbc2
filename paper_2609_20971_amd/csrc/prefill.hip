// Attention of all new tokens of a batch over a paged key-value cache: whole
// prompts, parts of prompts after what is cached already, a few drafted tokens;
// rows of any mixture in one call.
//
// Token i of the a new ones of a row of L tokens attends over keys 0 .. L - a + i.
// A tile is 128 queries of one row and one KV head, the group's heads of a token
// next to each other (16 tokens at a group of 8), so that all of them read the same
// keys and a tile's diagonal is short.  A workgroup's four waves have 32 queries
// each; keys come in blocks of 128.  S^T = K Q^T and O^T = V^T P^T on the 32x32x16
// matrix product in bf16, a query to a lane (softmax without exchanges but for one
// between the halves of a wave), Q in registers, K and V in LDS: 256-byte rows, 16-byte
// pieces swizzled so that reads have no bank conflicts, V read transposed.  BF16
// pages are copied to LDS directly, FP8 and FP4 ones through registers, widened
// once for all four waves (exact: E2M1 times a power of two, and E4M3, are bf16
// numbers; an FP8 head's factor goes into the softmax's scale and the result's).
// The next block's K is on its way during a block's softmax and second product, its V
// during the next first product.
//
// Bound by the matrix cores and the instructions around them for long rows, by the
// read of K and V for few queries.
//
// Sums are in fp32.  The weights go to the second product rounded once to bf16, and
// the denominator sums what goes there (on the matrix core), so that their common error
// cancels; the log-sum-exp, where it is asked for, has a sum of the weights before that.
//
// Work: unit u of a KV head is a tile, or where there are few tiles a piece of one,
// of at most P blocks of keys; pieces leave maximum, sum and weighted values in fp32,
// which a second launch joins in the order of the keys.  Lengths are on the GPU, so
// that every workgroup finds the units for itself.
#include <type_traits>

#include "attend_block.hpp"
#include "paged.hpp"

namespace rbs {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kBlock = 128;                      // queries of a tile, keys of a block
constexpr int kUnits = 1024;                     // pieces of a call whose tiles are split
constexpr int kPartFloats = kBlock * kHeadDim + 3 * kBlock;  // weighted values, maxima, sums of rounded and exact weights
constexpr int kMost = 1 << 29;                   // counts stop here

__device__ __forceinline__ int capped_add(int a, int b) { return min(a + b, kMost); }

// The rows, as kernel arguments of their own (scalar loads: a vector load of a page
// number would have to be waited for together with the copies on their way).
struct Rows {
  const int32_t* page_table;
  const int32_t* seq_lens;
  const int32_t* cu_tokens;
};
#define RBS_ROWS_ARGS \
  const int32_t *__restrict__ page_table, const int32_t *__restrict__ seq_lens, const int32_t *__restrict__ cu_tokens

struct RowWork {
  int tiles;   // 0: nothing to do
  int blocks;  // of the keys of its last token, at least 1
};

// What a row asks for.  Offsets are trusted like the page table: a row whose tokens
// are not inside Q has none.
__device__ __forceinline__ RowWork work_of_row(const PrefillArgs& a, int group, int begin, int end, int len) {
  RowWork w{0, 1};
  if (len < 0 || begin < 0 || end <= begin || end > a.n_tokens) return w;
  const int64_t cap = (int64_t)a.max_pages << a.cache.page_shift;
  w.tiles = (int)(((int64_t)(end - begin) * group + kBlock - 1) / kBlock);
  w.blocks = max(1, (int)((min((int64_t)len, cap) + kBlock - 1) / kBlock));
  return w;
}

// Where a workgroup keeps its plan.
struct Plan {
  int* first;   // [n_rows + 1]
  int* tiles;   // [n_rows], a thread's rows for itself
  int* blocks;
  int* sums;    // [4 kWaves]
};

// The units of a KV head: first[row] of them before the row, first[n_rows] in all, at
// most `piece` blocks to a unit; returns it.  Of the pieces that make at most `room`
// units the smallest is taken, from below (a count over the rows for each try, four
// at once); where there are as many tiles as that, whole tiles.
__device__ __forceinline__ int plan_units(const PrefillArgs& a, const Rows& rows, int room, const Plan& plan) {
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, group = a.n_q_heads / a.n_kv_heads;
  const int per = (a.n_rows + kThreads - 1) / kThreads;  // a thread's rows, one after another
  const int row0 = min(t * per, a.n_rows), row1 = min(row0 + per, a.n_rows);
  int* sums = plan.sums;
  int tiles = 0;
  float blocks = 0.f;  // (within 2^-12)
  bool descends = false;
  for (int r = row0; r < row1; ++r) {
    const int begin = rows.cu_tokens[r], end = rows.cu_tokens[r + 1];
    descends |= end < begin;
    const RowWork w = work_of_row(a, group, begin, end, rows.seq_lens[r]);
    plan.tiles[r] = w.tiles;
    plan.blocks[r] = w.blocks;
    tiles = capped_add(tiles, w.tiles);
    blocks += (float)w.tiles * w.blocks;
  }
  if (__syncthreads_or(descends)) {  // no offsets: rows may lie over each other
    for (int r = t; r <= a.n_rows; r += kThreads) plan.first[r] = 0;
    __syncthreads();
    return INT_MAX;
  }
  int piece = INT_MAX;
  if (room > 0) {
    // All tiles and all blocks.
    const int all = wave_scan(tiles, capped_add);
    for (int m = 1; m < 64; m *= 2) blocks += wave_xor_f(blocks, m);
    if (lane == 63) {
      sums[wave] = all;
      sums[kWaves + wave] = __float_as_int(blocks);
    }
    __syncthreads();
    int T = 0;
    float B = 0.f;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
      T = capped_add(T, sums[v]);
      B += __int_as_float(sums[kWaves + v]);
    }
    __syncthreads();
    T = __builtin_amdgcn_readfirstlane(T);
    if (T > 0 && T < room) {
      // (All the blocks over all the room: nothing smaller will do.  With a tile's last
      // piece as good as empty the second is enough.)
      const int least = __builtin_amdgcn_readfirstlane(max((int)fminf(B * 0.999f / room, (float)kMost), 1));
      const int enough = __builtin_amdgcn_readfirstlane((int)fminf(B * 1.001f / (room - T), (float)kMost) + 1);
      piece = enough;
      for (int p0 = least; p0 < enough && p0 < least + 8; p0 += 4) {
        int units[4] = {};
        for (int r = row0; r < row1; ++r) {
          const int n = plan.tiles[r], m = plan.blocks[r];
#pragma unroll
          for (int k = 0; k < 4; ++k) units[k] = capped_add(units[k], n * ((m + p0 + k - 1) / (p0 + k)));
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int x = wave_scan(units[k], capped_add);
          if (lane == 63) sums[k * kWaves + wave] = x;
        }
        __syncthreads();
        int found = 0;
#pragma unroll
        for (int k = 3; k >= 0; --k) {
          int U = 0;
#pragma unroll
          for (int v = 0; v < kWaves; ++v) U = capped_add(U, sums[k * kWaves + v]);
          if (U <= room) found = p0 + k;
        }
        __syncthreads();
        found = __builtin_amdgcn_readfirstlane(found);
        if (found > 0) {
          piece = found;
          break;
        }
      }
    }
  }
  if (piece != INT_MAX) {
    tiles = 0;
    for (int r = row0; r < row1; ++r) {
      const int n = plan.tiles[r] * ((plan.blocks[r] + piece - 1) / piece);
      plan.tiles[r] = n;
      tiles = capped_add(tiles, n);
    }
  }
  const int x = wave_scan(tiles, capped_add);
  if (lane == 63) sums[wave] = x;
  __syncthreads();
  int before = __builtin_amdgcn_update_dpp(0, x, 0x138, 0xf, 0xf, false), all = 0;  // wave_shr 1
#pragma unroll
  for (int v = 0; v < kWaves; ++v) {
    if (v == wave) before = capped_add(before, all);
    all = capped_add(all, sums[v]);
  }
  for (int r = row0; r < row1; ++r) {
    plan.first[r] = before;
    before = capped_add(before, plan.tiles[r]);
  }
  if (t == 0) plan.first[a.n_rows] = all;
  __syncthreads();
  return piece;
}

// A tile, or a piece of one.
struct Unit {
  int row, begin, tokens, len;  // the row's first token in Q, how many, and its cached tokens
  int tile, part, parts;        // of the row; of the tile
};

__device__ __forceinline__ Unit unit_of(const PrefillArgs& a, const Rows& rows, const int* first, int piece, int u) {
  const int group = a.n_q_heads / a.n_kv_heads;
  Unit n;
  n.row = __builtin_amdgcn_readfirstlane(seq_of(first, a.n_rows, u));
  const int local = __builtin_amdgcn_readfirstlane(u - first[n.row]);
  n.begin = rows.cu_tokens[n.row];
  n.tokens = rows.cu_tokens[n.row + 1] - n.begin;
  n.len = rows.seq_lens[n.row];
  const RowWork w = work_of_row(a, group, n.begin, n.begin + n.tokens, n.len);
  const int tiles = max(w.tiles, 1);
  n.parts = piece == INT_MAX ? 1 : (w.blocks + piece - 1) / piece;
  // The same keys for neighbours; the tiles with most keys first.
  n.part = local / tiles;
  n.tile = tiles - 1 - local % tiles;
  return n;
}

// Units are dealt out in bunches of neighbours, which read the same keys, to one XCD
// (workgroup j runs on XCD j % 8): bunch k of that XCD is bunch q = 8 k + x of all, of KV
// head q % H_kv.  Slot b of the launch gives KV head g and unit i of it (which may be
// past the last).
__device__ __forceinline__ void slot_of(int b, int n_kv_heads, int bunch, int* g, int* i) {
  const int x = b & 7, k = b >> 3;
  const int q = (k / bunch) * 8 + x;
  *g = q % n_kv_heads;
  *i = q / n_kv_heads * bunch + k % bunch;
}
__device__ __forceinline__ int bunch_of(int units, int n_kv_heads) {
  return max(1, min(8, (int)min((int64_t)units * n_kv_heads / 64, (int64_t)8)));
}
__device__ __forceinline__ int slots_of(int units, int n_kv_heads, int bunch) {
  const int64_t bunches = (int64_t)((units + bunch - 1) / bunch) * n_kv_heads;
  return (int)min((bunches + 7) / 8 * 8 * bunch, (int64_t)INT_MAX);
}

template <int kFmt>
constexpr int kCodeBytes = kFmt == kCacheFp4 ? kHeadDim / 2 : kFmt == kCacheFp8 ? kHeadDim : 2 * kHeadDim;

// A row's keys in the cache, for one wave's share of a block's copies.
template <int kFmt>
struct Pages {
  const int32_t* table;  // the row's
  int n_pages, shift, last_key;
  int64_t page_bytes;
  uint32_t tok_bytes;
  // Byte offset of 16 keys from j0 (a multiple of 16) on, of the last ones where j0 is past them.
  __device__ __forceinline__ int64_t at(int j0) const {
    const int j = __builtin_amdgcn_readfirstlane(min(j0, last_key & ~15));
    const int page = min(max(table[j >> shift], 0), n_pages - 1);
    return page * page_bytes + (int64_t)(j & ((1 << shift) - 1)) * tok_bytes;
  }
};

// One tensor's block in registers on its way to LDS (FP8, FP4).
template <int kFmt>
struct Staged {
  static constexpr int kLoads = kFmt == kCacheFp8 ? 4 : 2;
  static constexpr int kRows = kFmt == kCacheFp8 ? 8 : 16;  // of one load of a wave
  uint4 codes[kLoads];
  uint32_t scale[kLoads];
  // Load k of the wave has rows kRows (wave + 4 k) ..; 16 bytes to a lane.
  static __device__ __forceinline__ int row_of(int k) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    return kRows * (wave + kWaves * k) + lane / (64 / kRows);
  }
  __device__ __forceinline__ void load(const Pages<kFmt>& pages, const char* base, const char* scales, int block) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int piece = lane % (64 / kRows);
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      const int j0 = block * kBlock + kRows * (wave + kWaves * k), j16 = j0 & ~15;
      const int64_t at = pages.at(j16);
      // Keys past the row's last one: that one again.
      const int last = pages.last_key - min(j16, pages.last_key & ~15);
      const int r = j16 > pages.last_key ? last : min((j0 & 15) + lane / (64 / kRows), last);
      codes[k] = *reinterpret_cast<const uint4*>(base + at + (uint32_t)r * pages.tok_bytes + 16u * piece);
      if (kFmt == kCacheFp4) scale[k] = *reinterpret_cast<const uint8_t*>(scales + (at >> 4) + (uint32_t)r * (pages.tok_bytes >> 4) + piece);
    }
  }
  __device__ __forceinline__ void store(unsigned char* lds, bool is_v) const {
    const int piece = (threadIdx.x & 63) % (64 / kRows);
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      const int row = row_of(k);
      unsigned char* out = lds + row * 256;
      const uint32_t w[4] = {codes[k].x, codes[k].y, codes[k].z, codes[k].w};
      constexpr int kPieces = kFmt == kCacheFp8 ? 2 : 4;  // of 16 bytes
#pragma unroll
      for (int p = 0; p < kPieces; ++p) {
        const int c = kPieces * piece + p;
        uint4 v;
        if constexpr (kFmt == kCacheFp8) {
          uint32_t x[4];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            x[2 * e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w[2 * p + e], 1.f, false));
            x[2 * e + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w[2 * p + e], 1.f, true));
          }
          v = make_uint4(x[0], x[1], x[2], x[3]);
        } else {
          v = widen_e2m1(w[p], scale[k] << 23);
        }
        *reinterpret_cast<uint4*>(out + 16 * (is_v ? vswz(row, c) : kswz(row, c))) = v;
      }
    }
  }
};

template <int kFmt>
__device__ __forceinline__ float head_factor(const PrefillArgs& a, int head) {
  if (kFmt != kCacheFp8) return 1.f;
  const float m = a.cache.amax[head];
  return m > 0.f ? m / 448.f : 1.f;
}

// The result of a query: 64 of its elements in a lane.
__device__ __forceinline__ void write_query(const PrefillArgs& a, int head, int tok, int half, const f32x16* o, float m,
                                            float l, float l_exact, float v_factor) {
  const float inv = l > 0.f ? v_factor / l : l == 0.f ? 0.f : __builtin_nanf("");
  uint16_t* row = a.O + head * a.q_head + tok * a.q_tok;
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int rq = 0; rq < 4; ++rq)
      *reinterpret_cast<uint2*>(row + 32 * dt + 8 * rq + 4 * half) =
          make_uint2(two_bf16(o[dt][4 * rq] * inv, o[dt][4 * rq + 1] * inv),
                     two_bf16(o[dt][4 * rq + 2] * inv, o[dt][4 * rq + 3] * inv));
  if (a.lse != nullptr && half == 0)
    a.lse[(int64_t)head * a.n_tokens + tok] = l_exact == 0.f ? -INFINITY : (m + log2f(l_exact)) / kLog2e;
}

// What the workgroup's tiles in LDS are.
struct Tiles {
  unsigned char* k;
  unsigned char* v;
  int* bad;  // [kBlock]: the key's value is not finite
};

// Masked blocks: a weight of 0 times a value that is not finite would be NaN, so
// such values are taken out of the tile and added to the queries that attend them.
// (Weights are positive, so the sum is the same whatever they are.)
__device__ __forceinline__ void take_out(const Tiles& t, int limit, f32x16* o, int half) {
#pragma unroll 1
  for (int key = 0; key < kBlock; ++key) {
    if (__builtin_amdgcn_readfirstlane(t.bad[key]) == 0) continue;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int rq = 0; rq < 4; ++rq) {
        const int d = 32 * dt + 8 * rq + 4 * half;
        const uint2 w = *reinterpret_cast<const uint2*>(t.v + key * 256 + 16 * vswz(key, d >> 3) + 2 * (d & 7));
        const float x[4] = {bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y)};
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (key <= limit && !(fabsf(x[e]) < INFINITY)) o[dt][4 * rq + e] += x[e];
      }
  }
}

template <int kFmt, bool kLse>
__device__ __forceinline__ void attend_unit(const PrefillArgs& a, const Rows& rows, const Unit& n, int piece, int g, const Tiles& t,
                                            float* slot) {
  constexpr int KT = kBlock / 32;
  constexpr bool kCopied = kFmt == kCacheBf16;  // straight to LDS
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, l32 = lane & 31;
  const int group = a.n_q_heads / a.n_kv_heads;
  const int64_t queries = (int64_t)n.tokens * group, x0 = (int64_t)n.tile * kBlock;
  const int64_t cap = (int64_t)a.max_pages << a.cache.page_shift;
  const int before = n.len - n.tokens;  // position of the row's first new token
  const int held = (int)min((int64_t)n.len, cap);
  const int tile_last = min(before + (int)((min(x0 + kBlock, queries) - 1) / group), held - 1);
  const int first_last = min(before + (int)(x0 / group), held - 1);  // the last key of the tile's first query
  const int blocks = tile_last < 0 ? 0 : tile_last / kBlock + 1;
  const int b0 = piece == INT_MAX ? 0 : n.part * piece;
  const int b1 = piece == INT_MAX ? blocks : min(blocks, b0 + piece);
  const int plain = min(b1, (first_last + 1) / kBlock);  // blocks before it are attended whole

  // The lane's query (past the row's last one: that one, and not written).
  const int64_t x = x0 + 32 * wave + l32;
  const bool ok = x < queries;
  const int i = (int)((ok ? x : queries - 1) / group);
  const int head = g * group + (int)((ok ? x : queries - 1) - (int64_t)i * group), tok = n.begin + i;
  const int last = min(before + i, held - 1);  // its last key
  bf16x8 q[8];
  {
    const uint16_t* row = a.Q + head * a.q_head + tok * a.q_tok + 8 * half;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) q[ks] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(row + 16 * ks));
  }
  RBS_WAIT_VMCNT(0);  // (a wait for Q inside the loop would be one for the copies too)

  Pages<kFmt> pages;
  pages.table = rows.page_table + (int64_t)n.row * a.max_pages;
  pages.n_pages = a.cache.n_pages;
  pages.shift = a.cache.page_shift;
  pages.last_key = max(tile_last, 0);
  pages.page_bytes = a.cache.page * kCodeBytes<kFmt> / kHeadDim;
  pages.tok_bytes = (uint32_t)(a.cache.tok * kCodeBytes<kFmt> / kHeadDim);
  const int64_t head_bytes = g * a.cache.head * kCodeBytes<kFmt> / kHeadDim;
  const char* K = static_cast<const char*>(a.cache.K) + head_bytes;
  const char* V = static_cast<const char*>(a.cache.V) + head_bytes;
  const char* Ks = static_cast<const char*>(a.cache.K_scale) + g * a.cache.head / 32;
  const char* Vs = static_cast<const char*>(a.cache.V_scale) + g * a.cache.head / 32;
  const float scale_log2 = a.scale * kLog2e * head_factor<kFmt>(a, g);

  // BF16: the wave copies keys 32 wave .. + 31 of a block, in eight copies of four.  A
  // workgroup's copies all at once would hold its waves up at their issue, so that
  // half of a tensor's go out as its tile becomes free and the others in pairs among the
  // matrix and exponential steps.
  const uint32_t k_lds = __builtin_amdgcn_readfirstlane(lds_offset(t.k) + (uint32_t)wave * 8192u);
  const uint32_t v_lds = __builtin_amdgcn_readfirstlane(lds_offset(t.v) + (uint32_t)wave * 8192u);
  uint32_t k_off[4], v_off;
  {
    const int l4 = lane >> 4, pc = lane & 15;
#pragma unroll
    for (int j = 0; j < 4; ++j) k_off[j] = (uint32_t)(4 * j + l4) * pages.tok_bytes + 16u * (uint32_t)kswz(4 * j + l4, pc);
    v_off = (uint32_t)l4 * pages.tok_bytes + 16u * (uint32_t)vswz(l4, pc);
  }
  int64_t at_k[2], at_v[2];  // where the wave's two runs of 16 keys are, of the block whose K (V) is copied
  auto find = [&](int block) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < 2; ++h) at_k[h] = pages.at(block * kBlock + 32 * wave + 16 * h);
  };
  auto copy_pair = [&](bool is_v, int j) __attribute__((always_inline)) {  // copies j and j + 1 of 8
    const int64_t* from = is_v ? at_v : at_k;
#pragma unroll
    for (int c = j; c < j + 2; ++c) {
      const char* run = (is_v ? V : K) + from[c >> 2];
      lds_dma16(is_v ? run + (size_t)(4 * (c & 3)) * pages.tok_bytes : run, is_v ? v_off : k_off[c & 3],
                (is_v ? v_lds : k_lds) + 1024u * c);
    }
  };
  // Half of a block's copies, or where the row's last key is among its keys or before them, all: past it, that one again.
  auto copy_head = [&](int block, bool is_v) __attribute__((always_inline)) {
    const int64_t* from = is_v ? at_v : at_k;
    const int j0 = block * kBlock + 32 * wave;
    if (j0 + 31 <= pages.last_key) {
      copy_pair(is_v, 0);
      copy_pair(is_v, 2);
    } else {
#pragma unroll 1
      for (int c = 0; c < 8; ++c) {
        const int j16 = j0 + 16 * (c >> 2), r = 4 * (c & 3) + (lane >> 4);
        const int top = pages.last_key - min(j16, pages.last_key & ~15);
        const int row = j16 > pages.last_key ? top : min(r, top);
        const int at = is_v ? vswz(r, lane & 15) : kswz(r, lane & 15);
        lds_dma16((is_v ? V : K) + from[c >> 2], (uint32_t)row * pages.tok_bytes + 16u * (uint32_t)at,
                  (is_v ? v_lds : k_lds) + 1024u * c);
      }
    }
  };
  auto has_rest = [&](int block) __attribute__((always_inline)) { return block * kBlock + 32 * wave + 31 <= pages.last_key; };
  Staged<kCopied ? kCacheFp8 : kFmt> k_next, v_next;

  const int vq = (lane & 15) >> 2;
  const int vsub = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
  const int vbyte = 8 * (lane & 1);
  // Row m of the denominator's left operand takes the keys of lanes' halves of
  // parity m % 2: lane l finds its query's sum in element (l / 16) % 2 (attend_block.hpp).
  bf16x8 lsel;
  {
    const __bf16 one = (((lane >> 4) & 1) == (lane & 1)) ? (__bf16)1.0f : (__bf16)0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) lsel[e] = one;
  }
  f32x4 lacc{};
  auto l_of = [&]() __attribute__((always_inline)) { return ((lane >> 4) & 1) ? lacc[1] : lacc[0]; };
  float l_exact = 0.f;  // this half wave's, of the weights before their rounding
  bool is_nan = false;  // the lane's query has a weight that is NaN
  f32x16 o[4];
#pragma unroll
  for (int dt = 0; dt < 4; ++dt) o[dt] = f32x16{};
  float m = -INFINITY;

  auto attend = [&](auto masked_of, int b) __attribute__((always_inline)) {
    constexpr bool masked = decltype(masked_of)::value;
    const bool more = b + 1 < b1;
    if constexpr (kCopied) {
      RBS_WAIT_VMCNT(4);  // this block's K; its V may still be on its way
    } else {
      k_next.store(t.k, false);
    }
    __syncthreads();
    const bool v_rest = kCopied && b > b0 && has_rest(b);
    if (kCopied && more) find(b + 1);
    if constexpr (!kCopied)
      if (more) k_next.load(pages, K, Ks, b + 1);

    f32x16 s[KT];
#pragma unroll
    for (int mt = 0; mt < KT; ++mt) {
      s[mt] = f32x16{};
      const int row = 32 * mt + l32;
      const unsigned char* krow = t.k + row * 256;
#pragma unroll
      for (int ks = 0; ks < 8; ++ks) {
        const uint4 w = *reinterpret_cast<const uint4*>(krow + 16 * kswz(row, 2 * ks + half));
        s[mt] = mfma_bf16(__builtin_bit_cast(bf16x8, w), q[ks], s[mt]);
      }
      if (kCopied && mt < 2) {
        __builtin_amdgcn_sched_barrier(0);
        if (v_rest) copy_pair(true, 4 + 2 * mt);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    __syncthreads();  // every wave is done with this K
    const bool k_rest = kCopied && more && has_rest(b + 1);
    if constexpr (kCopied)
      if (more) copy_head(b + 1, false);
    const int limit = last - b * kBlock;  // the lane's last key in this block
    if constexpr (masked) {
#pragma unroll
      for (int mt = 0; mt < KT; ++mt) {
        const int lim = limit - 32 * mt - 4 * half;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[mt][r] = (8 * (r >> 2) + (r & 3)) > lim ? -INFINITY : s[mt][r];
          __builtin_amdgcn_sched_barrier(0);  // (64 compares' masks at once would not fit the scalar registers)
        }
      }
    }
    float top = -INFINITY;
#pragma unroll
    for (int mt = 0; mt < KT; ++mt)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, s[mt][r]);
    top = half_max(top) * scale_log2;
    if (__any(top > m + kRescaleSlack)) {
      // (Each query for itself: its result does not depend on the wave's others.)
      const float m_new = top > m + kRescaleSlack ? top : m;
      const float f = m_new == m ? 1.f : fast_exp2(m - m_new);
      m = m_new;
      l_exact *= f;
#pragma unroll
      for (int e = 0; e < 4; ++e) lacc[e] *= f;
#pragma unroll
      for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] *= f;
    }
    const float shift = m == -INFINITY ? 0.f : m;
    bf16x8 p[kBlock / 16];
#pragma unroll
    for (int mt = 0; mt < KT; ++mt) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[mt][r] = fast_exp2(fmaf(s[mt][r], scale_log2, -shift));
      if (kLse) {
        float sum[4] = {};
#pragma unroll
        for (int r = 0; r < 16; ++r) sum[r & 3] += s[mt][r];
        l_exact += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) p[2 * mt + (e >> 3)][e & 7] = (__bf16)s[mt][e];
      if (kCopied && mt < 2) {
        __builtin_amdgcn_sched_barrier(0);
        if (k_rest) copy_pair(false, 4 + 2 * mt);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    const f32x4 lacc_before = lacc;
#pragma unroll
    for (int c = 0; c < kBlock / 16; ++c) lacc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lsel, p[c], lacc, 0, 0, 0);
    if (__any(l_of() != l_of())) {
      // That product has two queries to a column, one of them times 0: a query with a
      // NaN takes no part in it.
#pragma unroll
      for (int c = 0; c < kBlock / 16; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) is_nan |= (float)p[c][e] != (float)p[c][e];
      is_nan = half_max(is_nan ? 1.f : 0.f) > 0.f;
      lacc = lacc_before;
#pragma unroll 1
      for (int again = 0; again < 1; ++again) {
#pragma unroll
        for (int c = 0; c < kBlock / 16; ++c) {
          const bf16x8 z{};
          lacc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lsel, is_nan ? z : p[c], lacc, 0, 0, 0);
        }
      }
    }
    if constexpr (kCopied) {
      if (more) RBS_WAIT_VMCNT(8); else RBS_WAIT_VMCNT(0);  // this block's V
    } else {
      v_next.store(t.v, true);
    }
    __syncthreads();
    if constexpr (!kCopied)
      if (more) v_next.load(pages, V, Vs, b + 1);
    if constexpr (masked) {
      // Does the block hold a value that is not finite?
      bool bad = false;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const uint4 w = *reinterpret_cast<const uint4*>(t.v + 16 * (tid + kThreads * k));
        const uint32_t z[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) bad |= (z[e] & 0x7f80u) == 0x7f80u || (z[e] & 0x7f800000u) == 0x7f800000u;
      }
      if (__syncthreads_or(bad)) {
        if (tid < kBlock) t.bad[tid] = 0;
        __syncthreads();
#pragma unroll 1
        for (int k = 0; k < 8; ++k) {
          const uint4 w = *reinterpret_cast<const uint4*>(t.v + 16 * (tid + kThreads * k));
          const uint32_t z[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if ((z[e] & 0x7f80u) == 0x7f80u || (z[e] & 0x7f800000u) == 0x7f800000u) t.bad[(tid + kThreads * k) >> 4] = 1;
        }
        __syncthreads();
        take_out(t, limit, o, half);
        __syncthreads();
#pragma unroll 1
        for (int k = 0; k < 8; ++k) {
          uint32_t* at = reinterpret_cast<uint32_t*>(t.v + 16 * (tid + kThreads * k));
          for (int e = 0; e < 4; ++e) {
            uint32_t z = at[e];
            if ((z & 0x7f80u) == 0x7f80u) z &= 0xffff0000u;
            if ((z & 0x7f800000u) == 0x7f800000u) z &= 0xffffu;
            at[e] = z;
          }
        }
        __syncthreads();
      }
    }
#pragma unroll
    for (int c = 0; c < kBlock / 16; ++c) {
      const int row0 = 16 * c + 4 * half + vq;
      const unsigned char* v0 = t.v + row0 * 256 + vbyte;
      const unsigned char* v1 = v0 + 8 * 256;
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) {
        const int pc = 16 * vswz(row0, 4 * dt + vsub);
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(v0 + pc));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(v1 + pc));
        bf16x8 v;
        __builtin_memcpy(&v, &lo, 8);
        __builtin_memcpy(reinterpret_cast<unsigned char*>(&v) + 8, &hi, 8);
        o[dt] = mfma_bf16(v, p[c], o[dt]);
      }
    }
    __syncthreads();  // every wave is done with this V
    if constexpr (kCopied) {
      if (more) {
        at_v[0] = at_k[0];
        at_v[1] = at_k[1];
        copy_head(b + 1, true);
      }
    }
  };

  if (b0 < b1) {
    if constexpr (kCopied) {
      find(b0);
      at_v[0] = at_k[0];
      at_v[1] = at_k[1];
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        copy_head(b0, v != 0);
        if (has_rest(b0)) {
          copy_pair(v != 0, 4);
          copy_pair(v != 0, 6);
        }
      }
    } else {
      k_next.load(pages, K, Ks, b0);
      v_next.load(pages, V, Vs, b0);
    }
  }
  int b = b0;
  for (; b < plain; ++b) attend(std::false_type{}, b);
  for (; b < b1; ++b) attend(std::true_type{}, b);

  if (x0 + 32 * wave >= queries) return;  // (no query of the wave's)
  const float l = is_nan ? __builtin_nanf("") : l_of();
  if (kLse) l_exact = half_sum(l_exact);
  if (n.parts == 1) {
    if (ok) write_query(a, head, tok, half, o, m, l, kLse ? l_exact : l, head_factor<kFmt>(a, a.n_kv_heads + g));
    return;
  }
  // A piece: every lane's 64 elements in runs of four, a KB for the wave at a time.
  if (b0 < b1) {
    float* out = slot + wave * 32 * kHeadDim;
#pragma unroll
    for (int k = 0; k < 16; ++k)
      *reinterpret_cast<float4*>(out + 4 * (64 * k + lane)) = make_float4(o[k >> 2][4 * (k & 3)], o[k >> 2][4 * (k & 3) + 1],
                                                                        o[k >> 2][4 * (k & 3) + 2], o[k >> 2][4 * (k & 3) + 3]);
  }
  if (half == 0) {
    float* sums = slot + kBlock * kHeadDim + 32 * wave + l32;
    sums[0] = m;
    sums[kBlock] = l;
    if (kLse) sums[2 * kBlock] = l_exact;
  }
}

template <int kFmt, bool kLse>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void paged_prefill_kernel(PrefillArgs a,
                                                                                                         int room,
                                                                                                         RBS_ROWS_ARGS) {
  const Rows rows{page_table, seq_lens, cu_tokens};
  __shared__ __align__(1024) unsigned char tiles[2 * kBlock * 256];
  __shared__ int sums[4 * kWaves], bad[kBlock];
  const Tiles t{tiles, tiles + kBlock * 256, bad};
  static_assert(sizeof(int) * (3 * kMaxRows + 1) <= sizeof(tiles), "the plan lies where the tiles will be");
  int* first = reinterpret_cast<int*>(tiles);
  const Plan plan{first, first + kMaxRows + 1, first + 2 * kMaxRows + 1, sums};
  for (int b = blockIdx.x;; b += gridDim.x) {
    const int piece = plan_units(a, rows, room, plan);
    const int units = __builtin_amdgcn_readfirstlane(first[a.n_rows]);
    const int bunch = bunch_of(units, a.n_kv_heads);
    if (b >= slots_of(units, a.n_kv_heads, bunch)) return;
    int g, i;
    slot_of(b, a.n_kv_heads, bunch, &g, &i);
    if (i < units) {
      const Unit n = unit_of(a, rows, first, piece, i);
      __syncthreads();  // every wave has read the offsets
      attend_unit<kFmt, kLse>(a, rows, n, piece, g, t, n.parts > 1 ? a.workspace + (size_t)(g * units + i) * kPartFloats : nullptr);
    }
    __syncthreads();  // the tiles are free
  }
}

// Joins the pieces of the tiles: a wave to 32 queries and 32 of their elements.
template <int kFmt>
__global__ __launch_bounds__(kThreads) void paged_prefill_join_kernel(PrefillArgs a, int room, RBS_ROWS_ARGS) {
  const Rows rows{page_table, seq_lens, cu_tokens};
  __shared__ int first[kMaxRows + 1], counts[2 * kMaxRows], sums[4 * kWaves];
  const int piece = plan_units(a, rows, room, Plan{first, counts, counts + kMaxRows, sums});
  if (piece == INT_MAX) return;
  const int units = __builtin_amdgcn_readfirstlane(first[a.n_rows]);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = lane >> 5, l32 = lane & 31;
  const int group = a.n_q_heads / a.n_kv_heads;
  // Workgroup (unit of all KV heads, 32 elements); only the first piece's of a tile stays.
  for (int b = blockIdx.x; b < units * a.n_kv_heads; b += gridDim.x) {
    const int g = b / units, i = b - g * units;
    const Unit n = unit_of(a, rows, first, piece, i);
    if (n.part != 0 || n.parts == 1) continue;
    const int tiles = (int)(((int64_t)n.tokens * group + kBlock - 1) / kBlock);
    const int64_t queries = (int64_t)n.tokens * group, x = (int64_t)n.tile * kBlock + 32 * wave + l32;
    if (x - l32 >= queries) continue;
    const int dt = blockIdx.y;
    const float* slots = a.workspace + (size_t)b * kPartFloats;
    const size_t step = (size_t)tiles * kPartFloats;
    const int at = kBlock * kHeadDim + 32 * wave + l32;
    float m = -INFINITY;
    for (int p = 0; p < n.parts; ++p) m = fmaxf(m, slots[p * step + at]);
    const float ref = m == -INFINITY ? 0.f : m;
    float l = 0.f, l_exact = 0.f;
    f32x16 o{};
    constexpr int kBatch = 4;
    for (int p0 = 0; p0 < n.parts; p0 += kBatch) {
      float pm[kBatch], pl[kBatch];
      float4 w[kBatch][4];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const float* slot = slots + min(p0 + k, n.parts - 1) * step;
        pm[k] = slot[at];
        pl[k] = slot[at + kBlock];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          w[k][e] = *reinterpret_cast<const float4*>(slot + wave * 32 * kHeadDim + 4 * (64 * (4 * dt + e) + lane));
      }
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        // (A piece without keys of the query's, or behind the tile's last block, which wrote no values.)
        if (p0 + k >= n.parts || pl[k] == 0.f) continue;
        const float f = fast_exp2(pm[k] - ref);
        l += pl[k] * f;
        if (a.lse != nullptr) l_exact += slots[(p0 + k) * step + at + 2 * kBlock] * f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          o[4 * e] += w[k][e].x * f;
          o[4 * e + 1] += w[k][e].y * f;
          o[4 * e + 2] += w[k][e].z * f;
          o[4 * e + 3] += w[k][e].w * f;
        }
      }
    }
    if (x >= queries) continue;
    const int tok_i = (int)(x / group), head = g * group + (int)(x - (int64_t)tok_i * group), tok = n.begin + tok_i;
    const float inv = l > 0.f ? head_factor<kFmt>(a, a.n_kv_heads + g) / l : l == 0.f ? 0.f : __builtin_nanf("");
    uint16_t* row = a.O + head * a.q_head + tok * a.q_tok + 32 * dt + 4 * half;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      *reinterpret_cast<uint2*>(row + 8 * e) = make_uint2(two_bf16(o[4 * e] * inv, o[4 * e + 1] * inv),
                                                          two_bf16(o[4 * e + 2] * inv, o[4 * e + 3] * inv));
    if (a.lse != nullptr && half == 0 && dt == 0)
      a.lse[(int64_t)head * a.n_tokens + tok] = l_exact == 0.f ? -INFINITY : (m + log2f(l_exact)) / kLog2e;
  }
}

template <int kFmt>
hipError_t launch(const PrefillArgs& a, hipStream_t s) {
  const int group = a.n_q_heads / a.n_kv_heads;
  // At most so many tiles of a KV head (of offsets that ascend; others are gone through in turns).
  const int64_t tiles = (int64_t)a.n_tokens * group / kBlock + (a.n_rows < a.n_tokens ? a.n_rows : a.n_tokens);
  const int64_t most = (int64_t)a.max_pages << a.cache.page_shift;  // keys of a row
  const int64_t units = tiles * a.n_kv_heads;
  const bool split = units < kUnits / 2 && most > kBlock;
  const int room = split ? kUnits / 2 / a.n_kv_heads : 0;
  const int64_t slots = (split ? kUnits : units) + 64 + 8 * a.n_kv_heads;
  const int grid = (int)(slots < (1 << 20) ? slots : (1 << 20));
  const auto kernel = a.lse != nullptr ? paged_prefill_kernel<kFmt, true> : paged_prefill_kernel<kFmt, false>;
  hipLaunchKernelGGL(kernel, dim3(grid), dim3(kThreads), 0, s, a, room, a.page_table, a.seq_lens, a.cu_tokens);
  if (split)
    hipLaunchKernelGGL(paged_prefill_join_kernel<kFmt>, dim3(kUnits / 2, 4), dim3(kThreads), 0, s, a, room, a.page_table,
                       a.seq_lens, a.cu_tokens);
  return hipGetLastError();
}

}  // namespace

size_t prefill_workspace_bytes() { return sizeof(float) * kUnits * kPartFloats; }

hipError_t launch_paged_prefill(const PrefillArgs& a, hipStream_t s) {
  switch (a.cache.format) {
    case kCacheBf16: return launch<kCacheBf16>(a, s);
    case kCacheFp8: return launch<kCacheFp8>(a, s);
    case kCacheFp4: return launch<kCacheFp4>(a, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace rbs
