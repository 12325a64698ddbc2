// Attention of one new token per row over a paged key-value cache.
//
// Bound by the read of K and V: each is read once, for all query heads of its KV
// head (4 H_q d flops for 4 H_kv d bytes a key: 8 flops a byte at a group of 8,
// where the card has 300).  So everything is arranged for loads in flight:
//
// - K and V go from memory to registers as matrix operands, with no LDS and no
//   barrier in the loop; a wave streams 32 keys at a time (64 in FP8, FP4) and asks for
//   the next ones, of the next row too, as soon as an operand has been used.
// - S^T = K Q^T and O^T = V^T P^T in 16x16x32 products with the (up to 16) query
//   heads of a KV head as columns.  Lane l holds column l % 16 of S and four keys
//   of each 16 (key_of), which is what the second product takes as its right
//   operand if V's rows come in the same order: P never leaves its lane.  V's
//   operand needs eight keys of one element; a lane has eight elements of eight
//   keys (16 lanes: whole rows) and regroups them with byte permutes.
// - A row's place in Q, O and lse is its number, or its last new token's where those
//   are packed: one scalar load as the row starts, and rows without one are skipped
//   like unused ones when the lengths are read.
// - The keys of all rows together are dealt out evenly: a tile is 32 (64) keys of
//   one row, and worker w of a KV head takes tiles [T w / W, T (w + 1) / W) of
//   the T tiles of all rows, its four waves every fourth of them.  Lengths are on
//   the GPU, so that every workgroup sums them up for itself.  A row that several
//   workers share is left in parts (maximum, sum, weighted values in fp32) that a
//   second launch joins, in the order of the workers: results do not depend on
//   which workgroup comes first.
//
// The exponentials' sum and the products are in fp32.  The weights go to the
// matrix core as two bf16 parts (the value and what its rounding left), off by
// 2^-16 together: in one part they would add about as much error as the result's
// own rounding, and the second product costs nothing here (160.3 us without it,
// 161.2 with it, 32 rows of 9000 to 16000 FP8 keys, 64 / 8 heads).
#include "paged.hpp"

namespace rbs {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
template <int kFmt>
constexpr bool is_fp8 = kFmt == kCacheFp8;
template <int kFmt>
constexpr bool is_fp4 = kFmt == kCacheFp4;
// Keys of one row that a wave takes at a time: 16 KB of K and V in bf16 and FP8, 8.5 in FP4.
template <int kFmt>
constexpr int kTile = kFmt == kCacheBf16 ? 32 : 64;
// Bytes of a head row of K or V: the codes, and with an FP4 row's four scales.
template <int kFmt>
constexpr int kCodeBytes = is_fp4<kFmt> ? kHeadDim / 2 : is_fp8<kFmt> ? kHeadDim : 2 * kHeadDim;
template <int kFmt>
constexpr int kRowBytes = kCodeBytes<kFmt> + (is_fp4<kFmt> ? kHeadDim / 32 : 0);
constexpr int kCols = 16;      // query heads of a unit
constexpr int kWorkers = 512;  // workgroups of a launch: two on each of 256 compute units
constexpr int kPartFloats = kCols * kHeadDim + 2 * kCols;  // weighted values, maxima, sums
// Rows of which the table holds at most so many tiles are a worker's alone, and there
// is no second launch.  In parts / whole, the GPU's time: one row of 384 keys 9.7 /
// 8.0 us, 64 rows of 200 to 256 15.6 / 14.2, to 384 16.2 / 16.7, to 500 17.4 / 19.4;
// FP8, 64 rows of 100 to 700 keys 16.4 / 16.0.
constexpr int kWholeTiles = 12;
// For few workgroups the launch that it saves (3 us of the calling thread) counts for
// more: one row of 700 keys on the GPU 9.5 / 11.1, called one by one 12.5 / 11.2.
constexpr int kWholeKeysOfFew = 768, kFewWhole = 8;
constexpr int kPad = kHeadDim + 4;  // floats between LDS rows (banks)
// A launch that reads more than this of K and V reads them past the caches: what
// it would leave there is gone before the next step reads it, and making room
// costs, most where the caches hold what others wrote.  Cached / past them, after a
// copy of 2 GB: 24 rows of up to 9000 keys (69 MB) 24.4 / 18.0 us, one of 20000
// (41 MB) 16.9 / 13.4, one of 131000 (268 MB) 76 / 46, 3000 (6 MB) 8.1 / 8.2; step
// after step, over more than the Infinity Cache, 32 rows of 9000 to 16000 keys
// (1.6 GB) 291 / 261, within it, 24 rows 20.6 / 22.0, 3000 11.0 / 12.0.  Not with
// more than 16 query heads to a KV head, whose units read the same keys (128
// heads: 190 / 223).
constexpr int64_t kCachedBytes = int64_t(16) << 20;
// Tiles that a row's start and end cost: with none of them a worker of many short
// rows comes late (24 rows of 1 to 9000 keys 28.4 us, 1: 23.4, 2 to 8: 21.3; 300
// rows of 10 to 600 keys 1: 33.7, 4: 30.3, 8: 32.8).
constexpr int kRowCost = 4;
// Rows are a wave's alone where no share is longer than kSoloShare, nor than
// kSoloRatio times an average wave's.  A workgroup's / a wave's: 300 rows of 10 to
// 100 FP8 keys, 4 KV heads, 18.3 / 14.9 us, 256 rows of 20 to 100, 8 / 8 heads, 20.7 /
// 18.1, 300 of 100 to 300 FP8 keys, 64 / 8, 37.5 / 35.9; longer rows 300 of 700 to 800,
// 64 / 8, 163 / 167; more different ones (a ratio of 3) 300 of 10 to 1000 64.9 / 73.9.
constexpr int kSoloShare = 20, kSoloRatio = 2;
// A join by single columns takes at most so many workgroups: one row of 20000 keys
// 18.2 us and not 20.8, of 131000 57 and not 60, 24 rows of 28 / 4 heads 20.6 and
// not 21.5; but 16 rows of 64 / 8 heads 29.9 and not 29.2, 64 rows of 32 / 4 72 and not
// 65.  Threads of a join's workgroup, 256 / 512 / 1024: one row of 2000 keys 9.5 /
// 10.9 / 12.4, 200 of 300 to 2000 41.9 / 43.3 / 46.3, one of 131000 50.1 / 50.1 / 51.5.
constexpr int kJoinThreads = 256, kFewJoins = 768;

// What the worker that has a row's first tile leaves for the join, at the
// workspace's end: one for each row and unit, or where there are more rows than
// workers, one for each worker (the row that goes on after it).
struct Shared {
  int row;    // -1: no row in parts
  int first;  // its first worker
  int last;   // and its last
  int slot;   // the first one's part, 0 or 1 (the others': 0)
};

struct Work {
  int units, tiles_of_cols, workers;  // KV heads x column tiles; workers of a unit
};

__host__ __device__ inline Work work_of_heads(int n_q_heads, int n_kv_heads) {
  const int group = n_q_heads / n_kv_heads;
  Work w;
  w.tiles_of_cols = (group + kCols - 1) / kCols;
  w.units = n_kv_heads * w.tiles_of_cols;
  w.workers = kWorkers / w.units > 1 ? kWorkers / w.units : 1;
  return w;
}

// The row's place in Q, O and lse (of a row that has one).
__device__ __forceinline__ int token_of(const int32_t* cu_tokens, int row) {
  return cu_tokens == nullptr ? row : cu_tokens[row + 1] - 1;
}
// Whether it has one.  Offsets are trusted like the page table: tokens outside Q are no row's.
__device__ __forceinline__ bool has_token(const int32_t* cu_tokens, int n_tokens, int row) {
  if (cu_tokens == nullptr) return true;
  const int begin = cu_tokens[row], end = cu_tokens[row + 1];
  return end > max(begin, 0) && end <= n_tokens;
}

// A row's share in the dealing out: its tiles, and kRowCost more for what it
// costs to start and end a row.
template <int kFmt>
__device__ __forceinline__ int share_of(int len) {
  return len > 0 ? (len - 1) / kTile<kFmt> + 1 + kRowCost : 0;
}

// first[row]: shares of the rows before it, first[n_rows]: of all; length[row] (-1:
// a row to leave alone); returns the longest share.  Each thread sums n_rows / 256 rows, then a scan over
// the threads.
template <int kFmt>
__device__ __forceinline__ int tile_offsets(const DecodeArgs& a, const int32_t* lens, const int32_t* cu_tokens,
                                             int* first, int* length, int* sums) {
  constexpr int kPer = kMaxRows / kThreads;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int per = (a.n_rows + kThreads - 1) / kThreads, row0 = t * per;
  const int64_t cap = (int64_t)a.max_pages << a.cache.page_shift;
  int share[kPer], mine = 0, longest = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) share[i] = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    if (i >= per) break;
    if (row0 + i < a.n_rows) {
      const int len = lens[row0 + i];
      const int clamped = has_token(cu_tokens, a.n_tokens, row0 + i) ? (int)(len < cap ? len : cap) : -1;
      length[row0 + i] = clamped;
      share[i] = share_of<kFmt>(clamped);
    }
    mine += share[i];
    longest = max(longest, share[i]);
  }
  const int x = wave_scan(mine, [](int u, int v) { return u + v; });
  longest = wave_scan(longest, [](int u, int v) { return max(u, v); });
  if (lane == 63) {
    sums[wave] = x;
    sums[kWaves + wave] = longest;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) longest = max(longest, sums[kWaves + w]);
  int before = x - mine;
#pragma unroll
  for (int w = 0; w < kWaves - 1; ++w) before += w < wave ? sums[w] : 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    if (i >= per) break;
    if (row0 + i < a.n_rows) first[row0 + i] = before;
    before += share[i];
  }
  if (t == kThreads - 1) first[a.n_rows] = before;
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(longest);
}

// The workers that share T tiles: each has at least a tile for each wave.
__device__ __forceinline__ int workers_of(int T, int workers) { return min(workers, (T + kWaves - 1) / kWaves); }
// Worker w of W starts at tile T w / W; the worker that tile t belongs to.
__device__ __forceinline__ int start_of(int T, int w, int W) { return (int)((int64_t)T * w / W); }
__device__ __forceinline__ int worker_of(int T, int t, int W) { return (int)(((int64_t)(t + 1) * W - 1) / T); }

__device__ __forceinline__ f32x4 mfma16(const uint4& a, const uint4& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                 0, 0);
}

// x combined over lanes l, l ^ 16, l ^ 32, l ^ 48.
template <typename Op>
__device__ __forceinline__ float over_rows(float x, Op op) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return op(__uint_as_float(s[0]), __uint_as_float(s[1]));
}

// bf16 of eight E4M3 codes (exact).
__device__ __forceinline__ uint4 widen(uint32_t lo, uint32_t hi) {
  auto pair = [](uint32_t w, bool top) __attribute__((always_inline)) {
    return top ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.f, true))
               : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.f, false));
  };
  return make_uint4(pair(lo, false), pair(lo, true), pair(hi, false), pair(hi, true));
}

__device__ __forceinline__ uint32_t word_of(const uint4& v, int i) {
  return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
}

// One wave's softmax state over the keys it has seen, for 16 query heads: o[i][r]
// is element 8 (4 (l / 16) + r) + i of column l % 16, in units of 2^m.
struct State {
  float m, l;
  f32x4 o[8];
};

template <int kFmt>
struct Tile {
  static constexpr int kSteps = kTile<kFmt> / 16;
  // Of 16 keys, with m = l % 16, c = l / 16.  bf16: key m, elements 32 x + 8 c ..;
  // FP8: key 8 x + m / 2, elements 64 (m % 2) + 16 c ..: eight lanes to a row of 128
  // bytes (in pieces of 64 200 rows of 300 to 2000 keys took 7% longer).
  uint4 k[kSteps][is_fp8<kFmt> ? 2 : 4];
  // bf16: key 4 c + x, elements 8 m ..; FP8: key 8 x + 2 c + m % 2, elements 16 (m / 2)
  // .., of which half is for the lane next to it: in loads of 8 bytes, each for its
  // own lane, a long read past the caches took 193 us and not 134.
  uint4 v[kSteps][is_fp8<kFmt> ? 2 : 4];
};

// FP4, of 16 keys: each load of the wave takes whole runs of memory (1 KB of K, 256
// bytes of V), and each scale is a byte of its own: 64 bytes for the wave.
template <>
struct Tile<kCacheFp4> {
  static constexpr int kSteps = kTile<kCacheFp4> / 16;
  uint4 k[kSteps];         // key 4 (m % 4) + m / 4, elements 32 c ..
  int k_scale[kSteps];     // of these 32 elements
  uint32_t v[kSteps][4];   // key 4 x + c, elements 8 m ..
  int v_scale[kSteps];     // of key 4 (m % 4) + c, elements 32 (m / 4) ..: what the four lanes of a quad need, one each
};

// Which of 16 keys a lane's logit (and weight) u is of, 0 <= u < 4.
template <int kFmt>
__device__ __forceinline__ int key_of(int c, int u) {
  return is_fp4<kFmt> ? 4 * u + c : is_fp8<kFmt> ? 8 * (u >> 1) + 2 * c + (u & 1) : 4 * c + u;
}

// 16 bytes of K or V; kOnce: without a place in the caches.
template <bool kOnce>
__device__ __forceinline__ uint4 load16(const char* p) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  if (!kOnce) return *reinterpret_cast<const uint4*>(p);
  const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
  return make_uint4(v.x, v.y, v.z, v.w);
}

template <bool kOnce>
__device__ __forceinline__ uint32_t load4(const char* p) {
  return kOnce ? __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(p)) : *reinterpret_cast<const uint32_t*>(p);
}
template <bool kOnce>
__device__ __forceinline__ int load1(const char* p) {
  return kOnce ? __builtin_nontemporal_load(reinterpret_cast<const uint8_t*>(p)) : *reinterpret_cast<const uint8_t*>(p);
}

// The other lane's of two next to each other.
__device__ __forceinline__ uint32_t neighbour(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xb1, 0xf, 0xf, false);  // quad_perm [1, 0, 3, 2]
}

// Lane u's of the lane's four.
__device__ __forceinline__ uint32_t of_quad(uint32_t x, int u) {
  const int i = (int)x;
  return (uint32_t)(u == 0   ? __builtin_amdgcn_update_dpp(0, i, 0x00, 0xf, 0xf, false)  // quad_perm [u, u, u, u]
                    : u == 1 ? __builtin_amdgcn_update_dpp(0, i, 0x55, 0xf, 0xf, false)
                    : u == 2 ? __builtin_amdgcn_update_dpp(0, i, 0xaa, 0xf, 0xf, false)
                             : __builtin_amdgcn_update_dpp(0, i, 0xff, 0xf, 0xf, false));
}

template <int kFmt>
struct Stream {
  const char* K;  // this KV head's
  const char* V;
  const char* K_scale;  // FP4: the scale of 32 elements at byte x of the codes is byte x / 16
  const char* V_scale;
  uint32_t ks_off, vs_off;
  int64_t page_bytes;
  int tok_bytes, n_pages, shift;
  uint32_t k_off, v_off;  // this lane's, within 16 keys
  bool once;              // see kCachedBytes

  // Byte offset of key j0 (a multiple of 16: within one page) of a row.  The page
  // number comes by a scalar load: a vector load's wait would be one for every key
  // and value on its way.
  __device__ __forceinline__ int64_t at(const int32_t* __restrict__ table, int len, int j0) const {
    const int page = min(max(table[__builtin_amdgcn_readfirstlane(min(j0, len - 1) >> shift)], 0), n_pages - 1);
    return page * page_bytes + (int64_t)(j0 & ((1 << shift) - 1)) * tok_bytes;
  }
  __device__ __forceinline__ void load_k(Tile<kFmt>& t, const int64_t* base) const {
    if (once) load_k_as<true>(t, base);
    else load_k_as<false>(t, base);
  }
  __device__ __forceinline__ void load_v(Tile<kFmt>& t, const int64_t* base) const {
    if (once) load_v_as<true>(t, base);
    else load_v_as<false>(t, base);
  }
  template <bool kOnce>
  __device__ __forceinline__ void load_k_as(Tile<kFmt>& t, const int64_t* base) const {
#pragma unroll
    for (int h = 0; h < Tile<kFmt>::kSteps; ++h) {
      if constexpr (is_fp4<kFmt>) {
        t.k[h] = load16<kOnce>(K + base[h] + k_off);
        t.k_scale[h] = load1<kOnce>(K_scale + (base[h] >> 4) + ks_off);
      } else {
#pragma unroll
        for (int x = 0; x < (is_fp8<kFmt> ? 2 : 4); ++x)
          t.k[h][x] = load16<kOnce>(K + base[h] + k_off + x * (is_fp8<kFmt> ? 8 * tok_bytes : 64));
      }
    }
  }
  template <bool kOnce>
  __device__ __forceinline__ void load_v_as(Tile<kFmt>& t, const int64_t* base) const {
#pragma unroll
    for (int h = 0; h < Tile<kFmt>::kSteps; ++h) {
      if constexpr (is_fp4<kFmt>) {
#pragma unroll
        for (int x = 0; x < 4; ++x) t.v[h][x] = load4<kOnce>(V + base[h] + v_off + 4 * x * tok_bytes);
        t.v_scale[h] = load1<kOnce>(V_scale + (base[h] >> 4) + vs_off);
      } else {
#pragma unroll
        for (int x = 0; x < (is_fp8<kFmt> ? 2 : 4); ++x)
          t.v[h][x] = load16<kOnce>(V + base[h] + v_off + x * (is_fp8<kFmt> ? 8 : 1) * tok_bytes);
      }
    }
  }
};

// One tile from key j on added to a wave's state; `next` gives the offsets of the
// tile to ask for (more: whether there is one).
template <int kFmt>
__device__ __forceinline__ void attend_tile(const Stream<kFmt>& st, Tile<kFmt>& tile, const uint4* q,
                                            float scale_log2, int j, int len, bool more, const int64_t* next,
                                            State& s) {
  constexpr int kSteps = Tile<kFmt>::kSteps;
  const int c = (threadIdx.x & 63) >> 4;
  const bool odd = threadIdx.x & 1;
  f32x4 sc[kSteps];
#pragma unroll
  for (int h = 0; h < kSteps; ++h) {
    if constexpr (is_fp4<kFmt>) {
      // Widened (exact).  The scaled product takes the codes as they are, with queries in two
      // 8-bit parts, but loses what lies 2^-14 under the largest of a few neighbouring
      // products (rows of 1 to 225 keys: lse off by 1e-6 of itself, 4e-8 here).  In time:
      // 8 rows of 139000 keys 138 us, 130 to 150 here; 32 of 9000 to 16384 87.4 both; one of 131071
      // 26.3, 25.1 here.
      sc[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < 4; ++x)
        sc[h] = mfma16(widen_e2m1(word_of(tile.k[h], x), (uint32_t)tile.k_scale[h] << 23), q[x], sc[h]);
    } else if constexpr (is_fp8<kFmt>) {
      // Rows 2 n and 2 n + 1 of the operand are the two halves of key n: the halves of
      // q with it in turn, of which every other row counts.
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const uint4 k0 = widen(tile.k[h][x].x, tile.k[h][x].y), k1 = widen(tile.k[h][x].z, tile.k[h][x].w);
        f32x4 lo{0.f, 0.f, 0.f, 0.f}, hi{0.f, 0.f, 0.f, 0.f};
        lo = mfma16(k0, q[0], lo);
        hi = mfma16(k0, q[2], hi);
        lo = mfma16(k1, q[1], lo);
        hi = mfma16(k1, q[3], hi);
        sc[h][2 * x] = lo[0] + hi[1];
        sc[h][2 * x + 1] = lo[2] + hi[3];
      }
    } else {
      sc[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < 4; ++x) sc[h] = mfma16(tile.k[h][x], q[x], sc[h]);
    }
  }
  if (more) st.load_k(tile, next);

  const bool partial = j + kTile<kFmt> > len;
  float x[4 * kSteps];
#pragma unroll
  for (int e = 0; e < 4 * kSteps; ++e) x[e] = sc[e >> 2][e & 3] * scale_log2;
  if (partial) {
#pragma unroll
    for (int e = 0; e < 4 * kSteps; ++e)
      if (j + 16 * (e >> 2) + key_of<kFmt>(c, e & 3) >= len) x[e] = -INFINITY;
  }
  float top = x[0];
#pragma unroll
  for (int e = 1; e < 4 * kSteps; ++e) top = fmaxf(top, x[e]);
  top = over_rows(top, [](float a, float b) { return fmaxf(a, b); });
  if (__any(top > s.m)) {
    const float m = fmaxf(s.m, top);
    const float keep = fast_exp2(s.m - (m == -INFINITY ? 0.f : m));
    s.m = m;
    s.l *= keep;
#pragma unroll
    for (int i = 0; i < 8; ++i) s.o[i] *= keep;
  }
  // (Logits of -inf alone, from infinite inputs, weigh nothing.)
  const float ref = s.m == -INFINITY ? 0.f : s.m;

#pragma unroll
  for (int b = 0; b < kSteps / 2; ++b) {  // 32 keys: the depth of a matrix product
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const float p0 = fast_exp2(x[8 * b + e] - ref), p1 = fast_exp2(x[8 * b + e + 1] - ref);
      s.l += p0 + p1;
      hi[e / 2] = two_bf16(p0, p1);
      lo[e / 2] = two_bf16(p0 - bf16_lo(hi[e / 2]), p1 - bf16_hi(hi[e / 2]));
    }
    const uint4 p_hi = make_uint4(hi[0], hi[1], hi[2], hi[3]), p_lo = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    uint4 v[8];
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const int h = 2 * b + (e >> 2);
      if constexpr (is_fp4<kFmt>) {
        const uint32_t scales = (uint32_t)tile.v_scale[h] << 23;
        v[e] = widen_e2m1(tile.v[h][e & 3], of_quad(scales, e & 3));
        v[e + 1] = widen_e2m1(tile.v[h][(e & 3) + 1], of_quad(scales, (e & 3) + 1));
      } else if constexpr (is_fp8<kFmt>) {
        const uint4& w = tile.v[h][(e >> 1) & 1];
        // (Every lane gives and takes: not inside a condition on the lane.)
        const uint32_t nx = neighbour(w.x), ny = neighbour(w.y), nz = neighbour(w.z), nw = neighbour(w.w);
        v[e] = widen(odd ? nz : w.x, odd ? nw : w.y);
        v[e + 1] = widen(odd ? w.z : nx, odd ? w.w : ny);
      } else {
        v[e] = tile.v[h][e & 3];
        v[e + 1] = tile.v[h][(e & 3) + 1];
      }
    }
    if (partial) {  // places past the row's length may hold anything, NaN too
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool in = j + 32 * b + 16 * (e >> 2) + key_of<kFmt>(c, e & 3) < len;
        v[e].x = in ? v[e].x : 0u;
        v[e].y = in ? v[e].y : 0u;
        v[e].z = in ? v[e].z : 0u;
        v[e].w = in ? v[e].w : 0u;
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t sel = (i & 1) ? 0x07060302u : 0x05040100u;
      uint32_t w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        w[k] = __builtin_amdgcn_perm(word_of(v[2 * k + 1], i >> 1), word_of(v[2 * k], i >> 1), sel);
      const uint4 op = make_uint4(w[0], w[1], w[2], w[3]);
      s.o[i] = mfma16(op, p_hi, s.o[i]);
      s.o[i] = mfma16(op, p_lo, s.o[i]);
    }
  }
  if (more) st.load_v(tile, next);
}

// The result of one column of a token: o holds 8 elements from 8 part on of the
// sum of weighted values, l the sum of weights in units of 2^m.
__device__ __forceinline__ void write_token(const DecodeArgs& a, int tok, int head, int part, const float* o,
                                            float m, float l, float v_scale) {
  const float f = v_scale / l;
  const uint4 w = make_uint4(two_bf16(o[0] * f, o[1] * f), two_bf16(o[2] * f, o[3] * f),
                             two_bf16(o[4] * f, o[5] * f), two_bf16(o[6] * f, o[7] * f));
  *reinterpret_cast<uint4*>(a.O + head * a.q_head + tok * a.q_tok + 8 * part) = w;
  if (part == 0 && a.lse != nullptr) a.lse[(int64_t)head * a.n_tokens + tok] = (m + __log2f(l)) * 0.69314718055994531f;
}

template <int kFmt>
__device__ __forceinline__ float value_scale(const DecodeArgs& a, int g) {
  if (!is_fp8<kFmt>) return 1.f;
  const float m = a.cache.amax[a.n_kv_heads + g];
  return m > 0.f ? m / 448.f : 1.f;
}

__device__ __forceinline__ Shared* shared_rows(const DecodeArgs& a) {
  return reinterpret_cast<Shared*>(a.workspace + (size_t)2 * kWorkers * kPartFloats);
}

// The first row whose share starts at x or after it (n_rows: none).
__device__ __forceinline__ int row_from(const int* first, int n_rows, int x) {
  int lo = 0, hi = n_rows;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] >= x) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

// kWhole: a row is one worker's, so that there is nothing to join.
template <int kFmt, bool kWhole>
__global__ __launch_bounds__(kThreads, 2) void paged_decode_kernel(
    DecodeArgs a, const int32_t* __restrict__ lens, const int32_t* __restrict__ page_table,
    const int32_t* __restrict__ cu_tokens) {
  __shared__ int first[kMaxRows + 1], length[kMaxRows], sums[2 * kWaves];
  __shared__ __align__(16) float acc[kWaves][kCols][kPad];
  __shared__ float ms[kWaves][kCols], ls[kWaves][kCols];
  const int lane = threadIdx.x & 63, c = lane >> 4, col = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Work wk = work_of_heads(a.n_q_heads, a.n_kv_heads);
  const int unit = blockIdx.x % wk.units, worker = blockIdx.x / wk.units;
  const int g = unit / wk.tiles_of_cols, group = a.n_q_heads / a.n_kv_heads;
  const int head0 = g * group + (unit % wk.tiles_of_cols) * kCols;
  const int cols = min(kCols, (g + 1) * group - head0);
  const int longest = tile_offsets<kFmt>(a, lens, cu_tokens, first, length, sums);
  const int T = first[a.n_rows];
  // Many short rows: each wave takes whole rows for itself, with nothing to join.
  const bool solo = longest <= kSoloShare && (int64_t)longest * (kWaves * wk.workers) <= (int64_t)kSoloRatio * T;
  const int W = solo ? kWaves * wk.workers : workers_of(T, wk.workers), id = solo ? kWaves * worker + wave : worker;
  int t = id < W ? start_of(T, id, W) : T, t_end = id < W ? start_of(T, id + 1, W) : T;
  if (kWhole || solo) {
    t = __builtin_amdgcn_readfirstlane(first[row_from(first, a.n_rows, t)]);
    t_end = __builtin_amdgcn_readfirstlane(first[row_from(first, a.n_rows, t_end)]);
  }
  const int step = solo ? 1 : kWaves, offset = solo ? 0 : wave;
  const bool by_row = a.n_rows <= wk.workers;
  Shared shared{-1, 0, 0, 0};

  // Empty rows: zeros, and -inf.
  for (int row = worker; row < a.n_rows; row += wk.workers) {
    if (length[row] != 0) continue;
    const int tok = token_of(cu_tokens, row);
    for (int x = threadIdx.x; x < cols * (kHeadDim / 8); x += kThreads)
      *reinterpret_cast<uint4*>(a.O + (head0 + x / 16) * a.q_head + tok * a.q_tok + 8 * (x % 16)) =
          make_uint4(0u, 0u, 0u, 0u);
    if (a.lse != nullptr && (int)threadIdx.x < cols)
      a.lse[(int64_t)(head0 + threadIdx.x) * a.n_tokens + tok] = -INFINITY;
  }

  constexpr int kSteps = Tile<kFmt>::kSteps;
  // Bytes of so many elements.
  auto bytes = [](int64_t x) __attribute__((always_inline)) { return x * kCodeBytes<kFmt> / kHeadDim; };
  Stream<kFmt> st;
  st.K = static_cast<const char*>(a.cache.K) + bytes(g * a.cache.head);
  st.V = static_cast<const char*>(a.cache.V) + bytes(g * a.cache.head);
  st.page_bytes = bytes(a.cache.page);
  st.tok_bytes = (int)bytes(a.cache.tok);
  st.n_pages = a.cache.n_pages;
  st.shift = a.cache.page_shift;
  st.once = wk.tiles_of_cols == 1 && (int64_t)T * wk.units * (kTile<kFmt> * 2 * kRowBytes<kFmt>) >= kCachedBytes;
  st.k_off = is_fp8<kFmt> ? (col >> 1) * st.tok_bytes + 64 * (col & 1) + 16 * c : col * st.tok_bytes + 16 * c;
  st.v_off = is_fp8<kFmt> ? (2 * c + (col & 1)) * st.tok_bytes + 16 * (col >> 1) : 4 * c * st.tok_bytes + 16 * col;
  if constexpr (is_fp4<kFmt>) {
    st.K_scale = static_cast<const char*>(a.cache.K_scale) + g * a.cache.head / 32;
    st.V_scale = static_cast<const char*>(a.cache.V_scale) + g * a.cache.head / 32;
    st.k_off = (4 * (col & 3) + (col >> 2)) * st.tok_bytes + 16 * c;
    st.v_off = c * st.tok_bytes + 4 * col;
    st.ks_off = (4 * (col & 3) + (col >> 2)) * (st.tok_bytes >> 4) + c;
    st.vs_off = (4 * (col & 3) + c) * (st.tok_bytes >> 4) + (col >> 2);
  }
  float scale_log2 = a.scale * kLog2e;
  if (is_fp8<kFmt> && a.cache.amax[g] > 0.f) scale_log2 *= a.cache.amax[g] / 448.f;
  const float v_scale = value_scale<kFmt>(a, g);

  // The wave's next tile: tile `tile` of row `row` (-1: none), of `len` keys.  It
  // runs ahead of the rows below by one tile, whose keys and values are on their
  // way.
  struct Cursor {
    int row, tile, end, len;  // end: of the row's share
  } next{-1, 0, 0, 0};
  // Moves the cursor to the wave's first tile in row r or after it: the wave takes
  // tiles offset, offset + step, .. of each row's share.
  auto seek = [&](int r) __attribute__((always_inline)) {
    for (;; ++r) {
      if (r >= a.n_rows || first[r] >= t_end) {
        next.row = -1;
        return;
      }
      const int x = max(first[r], t) + offset, to = min(first[r + 1] - kRowCost, t_end);
      if (x < to) {
        next.row = __builtin_amdgcn_readfirstlane(r);
        next.tile = __builtin_amdgcn_readfirstlane(x - first[r]);
        next.end = __builtin_amdgcn_readfirstlane(to - first[r]);
        next.len = __builtin_amdgcn_readfirstlane(length[next.row]);
        return;
      }
      if (first[r + 1] == first[r]) r = seq_of(first, a.n_rows, first[r]) - 1;  // past all the empty rows here
    }
  };
  auto offsets = [&](int64_t* base) __attribute__((always_inline)) {
    const int32_t* table = page_table + (int64_t)__builtin_amdgcn_readfirstlane(next.row) * a.max_pages;
    const int len = __builtin_amdgcn_readfirstlane(next.len);
    const int j = __builtin_amdgcn_readfirstlane(next.tile * kTile<kFmt>);
#pragma unroll
    for (int h = 0; h < kSteps; ++h) base[h] = st.at(table, len, j + 16 * h);
  };
  int row = t < t_end ? seq_of(first, a.n_rows, t) : 0;
  Tile<kFmt> tile;
  if (t < t_end) seek(row);
  if (next.row >= 0) {
    int64_t base[kSteps];
    offsets(base);
    st.load_k(tile, base);
    st.load_v(tile, base);
  }
  int at = t;  // the first tile that is still to do
  bool is_first = true;
  while (at < t_end) {
    if (first[row + 1] <= at && first[++row + 1] <= at) row = seq_of(first, a.n_rows, at);
    const int r = __builtin_amdgcn_readfirstlane(row);
    const int last = first[r + 1] - kRowCost;  // past the row's last tile
    if (at >= last) {
      at = first[r + 1];
      continue;
    }
    const int stop = min(last, t_end);
    const bool begins = at == first[r], whole = begins && stop == last;
    const int tok = token_of(cu_tokens, r);
    uint4 q[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      // Elements that the K operand's lane holds.
      const int d = is_fp4<kFmt> ? 32 * c + 8 * x : is_fp8<kFmt> ? 64 * (x >> 1) + 16 * c + 8 * (x & 1) : 32 * x + 8 * c;
      q[x] = make_uint4(0u, 0u, 0u, 0u);
      if (col < cols) q[x] = *reinterpret_cast<const uint4*>(a.Q + (head0 + col) * a.q_head + tok * a.q_tok + d);
    }
    // Waited for here: in the loop the wait for the first Q would be one for the
    // values on their way as well, at every tile.
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
    State s;
    s.m = -INFINITY;
    s.l = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s.o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    while (next.row == r) {
      const int j = next.tile * kTile<kFmt>, len = next.len;
      next.tile += step;
      if (next.tile >= next.end) seek(r + 1);
      int64_t base[kSteps] = {};
      if (next.row >= 0) offsets(base);
      attend_tile<kFmt>(st, tile, q, scale_log2, j, len, next.row >= 0, base, s);
    }
    s.l = over_rows(s.l, [](float a, float b) { return a + b; });

    if (solo) {
      if (col < cols) {
        const float f = v_scale / s.l;
        uint16_t* out = a.O + (head0 + col) * a.q_head + tok * a.q_tok + 32 * c;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          *reinterpret_cast<uint4*>(out + 8 * e) =
              make_uint4(two_bf16(s.o[0][e] * f, s.o[1][e] * f), two_bf16(s.o[2][e] * f, s.o[3][e] * f),
                         two_bf16(s.o[4][e] * f, s.o[5][e] * f), two_bf16(s.o[6][e] * f, s.o[7][e] * f));
        if (c == 0 && a.lse != nullptr)
          a.lse[(int64_t)(head0 + col) * a.n_tokens + tok] = (s.m + __log2f(s.l)) * 0.69314718055994531f;
      }
      if (!kWhole && by_row && lane == 0) shared_rows(a)[r * wk.units + unit] = Shared{-1, 0, 0, 0};
      at = first[r + 1];
      continue;
    }

    // The four waves' states joined.
    if (c == 0) {
      ms[wave][col] = s.m;
      ls[wave][col] = s.l;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float* at = &acc[wave][col][8 * (4 * c + e)];
      *reinterpret_cast<float4*>(at) = make_float4(s.o[0][e], s.o[1][e], s.o[2][e], s.o[3][e]);
      *reinterpret_cast<float4*>(at + 4) = make_float4(s.o[4][e], s.o[5][e], s.o[6][e], s.o[7][e]);
    }
    __syncthreads();
    const int hc = threadIdx.x >> 4, part = threadIdx.x & 15;
    if (hc < cols) {
      float m = ms[0][hc], l = 0.f, o[8] = {};
#pragma unroll
      for (int w = 1; w < kWaves; ++w) m = fmaxf(m, ms[w][hc]);
      const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = fast_exp2(ms[w][hc] - ref);
        l += ls[w][hc] * f;
        const float4 x = *reinterpret_cast<const float4*>(&acc[w][hc][8 * part]);
        const float4 y = *reinterpret_cast<const float4*>(&acc[w][hc][8 * part + 4]);
        o[0] += x.x * f; o[1] += x.y * f; o[2] += x.z * f; o[3] += x.w * f;
        o[4] += y.x * f; o[5] += y.y * f; o[6] += y.z * f; o[7] += y.w * f;
      }
      if (kWhole || whole) {
        write_token(a, tok, head0 + hc, part, o, m, l, v_scale);
      } else {
        float* slot = a.workspace + (size_t)(2 * blockIdx.x + (is_first ? 0 : 1)) * kPartFloats;
        *reinterpret_cast<float4*>(slot + hc * kHeadDim + 8 * part) = make_float4(o[0], o[1], o[2], o[3]);
        *reinterpret_cast<float4*>(slot + hc * kHeadDim + 8 * part + 4) = make_float4(o[4], o[5], o[6], o[7]);
        if (part == 0) {
          slot[kCols * kHeadDim + hc] = m;
          slot[kCols * kHeadDim + kCols + hc] = l;
        }
      }
    }
    __syncthreads();
    if (!kWhole && begins) {
      shared = Shared{whole ? -1 : r, worker, worker_of(T, last - 1, W), is_first ? 0 : 1};
      if (by_row && threadIdx.x == 0) shared_rows(a)[r * wk.units + unit] = shared;
    }
    is_first = false;
    at = first[r + 1];
  }
  if (!kWhole && !by_row && threadIdx.x == 0) shared_rows(a)[blockIdx.x] = shared;
}

// Joins the parts of a row.  16 threads take a column's 128 elements, and as many
// sets of 16 as there are threads for take every so many-th part; eight parts'
// loads are in flight at a time (a row of 128K keys has 128 parts).  One column to
// a workgroup where that makes few of them, otherwise four: most workgroups of a
// large batch find nothing to join.
template <int kFmt, int kJoinCols>
__global__ __launch_bounds__(kJoinThreads) void paged_decode_join_kernel(DecodeArgs a) {
  constexpr int kSets = kJoinThreads / 16, kBatch = kJoinCols == 1 ? 4 : 8;
  __shared__ __align__(16) float acc[kSets][kPad];
  __shared__ float ms[kSets], ls[kSets];
  const Work wk = work_of_heads(a.n_q_heads, a.n_kv_heads);
  const bool by_row = a.n_rows <= wk.workers;
  const int unit = blockIdx.x % wk.units;
  const Shared shared = shared_rows(a)[blockIdx.x];
  const int row = blockIdx.x / wk.units;
  // (A row of no length or no token is no worker's: there is no record of it.)
  if (by_row && (a.seq_lens[row] <= 0 || !has_token(a.cu_tokens, a.n_tokens, row))) return;
  if (shared.row < 0) return;
  const int wa = shared.first;
  const int g = unit / wk.tiles_of_cols, group = a.n_q_heads / a.n_kv_heads;
  const int head0 = g * group + (unit % wk.tiles_of_cols) * kCols;
  const int col0 = blockIdx.y * kJoinCols, cols = min(kJoinCols, min(kCols, (g + 1) * group - head0) - col0);
  if (cols <= 0) return;
  const int set = threadIdx.x >> 4, part = threadIdx.x & 15;
  const int sets_each = kSets / cols, hc = set % cols, mine = set / cols;  // (sets past cols * sets_each are idle)
  const int parts = shared.last - wa + 1;
  const float* base = a.workspace + (size_t)2 * (wa * wk.units + unit) * kPartFloats;
  float m = -INFINITY, l = 0.f, o[8] = {};
  if (mine < sets_each) {
    for (int p0 = mine; p0 < parts; p0 += kBatch * sets_each) {
      float pm[kBatch], pl[kBatch];
      float4 x[kBatch], y[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const int p = min(p0 + i * sets_each, parts - 1);
        const float* slot = base + (size_t)(2 * p * wk.units + (p == 0 ? shared.slot : 0)) * kPartFloats;
        pm[i] = slot[kCols * kHeadDim + col0 + hc];
        pl[i] = slot[kCols * kHeadDim + kCols + col0 + hc];
        x[i] = *reinterpret_cast<const float4*>(slot + (col0 + hc) * kHeadDim + 8 * part);
        y[i] = *reinterpret_cast<const float4*>(slot + (col0 + hc) * kHeadDim + 8 * part + 4);
      }
      float top = m;
#pragma unroll
      for (int i = 0; i < kBatch; ++i) top = fmaxf(top, pm[i]);
      const float ref = top == -INFINITY ? 0.f : top, keep = fast_exp2(m - ref);
      m = top;
      l *= keep;
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] *= keep;
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        if (p0 + i * sets_each >= parts) break;
        const float f = fast_exp2(pm[i] - ref);
        l += pl[i] * f;
        o[0] += x[i].x * f; o[1] += x[i].y * f; o[2] += x[i].z * f; o[3] += x[i].w * f;
        o[4] += y[i].x * f; o[5] += y[i].y * f; o[6] += y[i].z * f; o[7] += y[i].w * f;
      }
    }
  }
  if (part == 0) {
    ms[set] = m;
    ls[set] = l;
  }
  *reinterpret_cast<float4*>(&acc[set][8 * part]) = make_float4(o[0], o[1], o[2], o[3]);
  *reinterpret_cast<float4*>(&acc[set][8 * part + 4]) = make_float4(o[4], o[5], o[6], o[7]);
  __syncthreads();
  if (mine > 0) return;
  float top = m;
  for (int i = 1; i < sets_each; ++i) top = fmaxf(top, ms[hc + i * cols]);
  const float ref = top == -INFINITY ? 0.f : top;
  float sum = 0.f, out[8] = {};
  for (int i = 0; i < sets_each; ++i) {
    const float f = fast_exp2(ms[hc + i * cols] - ref);
    sum += ls[hc + i * cols] * f;
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] += acc[hc + i * cols][8 * part + e] * f;
  }
  write_token(a, token_of(a.cu_tokens, shared.row), head0 + col0 + hc, part, out, top, sum, value_scale<kFmt>(a, g));
}

template <int kFmt>
hipError_t launch(const DecodeArgs& a, hipStream_t s) {
  const Work wk = work_of_heads(a.n_q_heads, a.n_kv_heads);
  const int group = a.n_q_heads / a.n_kv_heads, cols = group < kCols ? group : kCols;
  const dim3 grid(wk.units * wk.workers);
  const int64_t most = (int64_t)a.max_pages << a.cache.page_shift;  // keys of a row
  if (most <= kWholeTiles * kTile<kFmt> || (most <= kWholeKeysOfFew && a.n_rows * wk.units <= kFewWhole)) {
    hipLaunchKernelGGL((paged_decode_kernel<kFmt, true>), grid, dim3(kThreads), 0, s, a, a.seq_lens, a.page_table,
                       a.cu_tokens);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((paged_decode_kernel<kFmt, false>), grid, dim3(kThreads), 0, s, a, a.seq_lens, a.page_table,
                       a.cu_tokens);
  const int joins = wk.units * (a.n_rows < wk.workers ? a.n_rows : wk.workers);
  if (joins * cols <= kFewJoins)
    hipLaunchKernelGGL((paged_decode_join_kernel<kFmt, 1>), dim3(joins, cols), dim3(kJoinThreads), 0, s, a);
  else
    hipLaunchKernelGGL((paged_decode_join_kernel<kFmt, 4>), dim3(joins, (cols + 3) / 4), dim3(kJoinThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

// Two parts for each worker; the workers of all units are kWorkers at most, or
// one for each unit (units <= query heads).
size_t decode_workspace_bytes() { return sizeof(float) * 2 * kWorkers * kPartFloats + kWorkers * sizeof(Shared); }

hipError_t launch_paged_decode(const DecodeArgs& a, hipStream_t s) {
  switch (a.cache.format) {
    case kCacheBf16: return launch<kCacheBf16>(a, s);
    case kCacheFp8: return launch<kCacheFp8>(a, s);
    case kCacheFp4: return launch<kCacheFp4>(a, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace rbs
