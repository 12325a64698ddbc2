// Attention of all new tokens of a batch over a paged key-value cache: whole
// prompts, parts of prompts after what is cached already, a few drafted tokens;
// rows of any mixture in one call.
//
// Token i of the a new ones of a row of L tokens attends over keys 0 .. L - a + i.
// A tile is 128 queries of one row and one KV head, the group's heads of a token
// next to each other (16 tokens at a group of 8), so that all of them read the same
// keys and a tile's diagonal is short.  A workgroup's four waves have 32 queries
// each (of a row of at most 32 queries all of them, and every fourth block of keys each:
// attend_few); keys come in blocks of 64.  S^T = K Q^T and O^T = V^T P^T on the 32x32x16
// matrix product in bf16, a query to a lane (softmax without exchanges but for one
// between the halves of a wave), Q in registers, K and V in LDS, two blocks of each: 256-byte
// rows, 16-byte pieces swizzled so that reads have no bank conflicts, V read transposed.
// BF16 pages are copied to LDS directly, FP8 and FP4 ones through registers, widened
// once for all four waves (exact: E2M1 times a power of two, and E4M3, are bf16
// numbers; an FP8 head's factor goes into the softmax's scale and the result's).
//
// Long rows are bound by the matrix cores and the instructions between their products:
// 2048 tokens after 65536, 32 heads on 4, take 1.95 to 2.03 ms in every format (1145 to 1100
// TFLOP/s; a library product of 16384^3 reaches 1350).  BF16: the cores are busy 58 % of the
// cycles at a clock that such work lowers to 1.7 to 1.8 GHz (16384 tokens).  FP4: 50 % at
// 1.9, with bank conflicts of the widened V's way into LDS in a quarter of the cycles.  Few queries are
// bound by what a unit takes before its first and after its last block.
//
// Sums are in fp32.  A tile's weights go to the second product rounded once to bf16, and
// the denominator sums what goes there, so that their common error cancels; the
// log-sum-exp, where it is asked for, has a sum of the weights before that.  (A second
// part would be half as much again of the products that bound it; the result is off from 64 bits by
// 0.00193 of itself in the root mean square, its own rounding by 0.00167.)  Rows of at most 32
// queries have the weights in two parts, as the decode calls do, so that a token that is
// checked and one that is decoded differ by the rounding of the result.
//
// Work: unit u of a KV head is a tile, or where there are few tiles a piece of one,
// of at most P blocks of keys; pieces leave maximum, sums and weighted values in fp32,
// which a second launch joins in the order of the keys.  Lengths are on the GPU, so
// that every workgroup finds the units for itself.
#include <type_traits>

#include "attend_block.hpp"
#include "paged.hpp"

namespace rbs {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kQueries = 128;                    // of a tile
constexpr int kKeys = 64;                        // of a block
constexpr int kFewQueries = 32;                  // a row's, up to which its keys are divided among the waves
constexpr int kBlockBytes = kKeys * 2 * kHeadDim;  // of K or V in LDS
// Pieces of a call whose tiles are split: two workgroups to a CU.  512 tokens after 8192
// take 94 us, 102 at 256 pieces and 106 at 1024; 32 rows of 4 drafted tokens after 16000 in
// FP4 114, 155 and 122; 1 token after 65535 44, 41 and 55.
constexpr int kUnits = 512;
// Blocks of a piece, at least.  4 tokens after 16384 in FP4 take 20.4 us, 22.8 with pieces of 2;
// 128 after 1024 20.6 and 21.7, 1 after 3000 14.6 and 14.0.
constexpr int kLeast = 4;
constexpr int kPartFloats = kQueries * kHeadDim + 3 * kQueries;  // weighted values, maxima, sums of rounded and exact weights

// Division of 32-bit numbers by one that the host knows, by a product with its
// reciprocal (Granlund and Montgomery 1994): the quotient is exact.
struct Divisor {
  uint32_t d, m, s1, s2;
  explicit Divisor(uint32_t d_) : d(d_) {
    uint32_t l = 0;
    while ((uint64_t(1) << l) < d) ++l;
    m = (uint32_t)(((uint64_t(1) << 32) * ((uint64_t(1) << l) - d)) / d + 1);
    s1 = l < 1 ? l : 1;
    s2 = l < 1 ? 0 : l - 1;
  }
  __device__ __forceinline__ uint32_t of(uint32_t x) const {
    const uint32_t t = __umulhi(m, x);
    return (t + ((x - t) >> s1)) >> s2;
  }
};
// (A call's queries of a KV head are fewer than 2^30.)
struct Heads {
  Divisor group, n_kv;
};

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
  w.tiles = (int)(((uint32_t)(end - begin) * (uint32_t)group + kQueries - 1) / kQueries);
  w.blocks = max(1, (int)((min((int64_t)len, cap) + kKeys - 1) / kKeys));
  return w;
}

// What is to do, found by every workgroup for itself.  A KV head's units are numbered
// row after row; of a row by pieces, so that neighbours read the same keys, and of a
// piece by tiles, those with most keys first.
//
// The pieces: at most so many blocks to a unit that there are at most `room` units, the
// smallest such number, tried from below four at a time (a count over the rows for
// each); where there are as many tiles as that, whole tiles.  It is found by the first
// launch (known: 0) and left for the join, which derives the rest from it in whole numbers: the
// rule's floats, compiled a second time, could round another way.
__device__ __forceinline__ int pieces_of(int blocks, int piece) {
  return piece == INT_MAX ? 1 : (blocks + piece - 1) / piece;
}

// The numbers to try, given all tiles and all blocks of them (within 2^-12).
struct Tries {
  int least, enough;  // nothing smaller will do; with each tile's last piece as good as empty this will
};
__device__ __forceinline__ Tries tries_of(int tiles, float blocks, int room) {
  Tries t;
  t.least = __builtin_amdgcn_readfirstlane(max((int)fminf(blocks * 0.999f / room, (float)kMost), kLeast));
  t.enough = max(__builtin_amdgcn_readfirstlane((int)fminf(blocks * 1.001f / (room - tiles), (float)kMost) + 1), kLeast);
  return t;
}

// Whether pieces are worth their join: what the longest row's tiles save by them against
// the join, in the time of a block by itself (1.24 us; beside another workgroup's 2).  A join
// is a launch and the parts' way through memory.  Whole and in pieces: 1024 tokens 30 and
// 41 us, 1024 after 2048 67 and 72, 1024 after 8192 177 and 164, 64 after 2048 45 and 20.
__device__ __forceinline__ bool worth(float longest, int piece, int64_t units) {
  const float u = (float)units, beside = fminf(fmaxf(u * (2.f / kUnits) - 1.f, 0.f), 1.f);
  return __builtin_amdgcn_readfirstlane(longest - (float)piece * (1.f + 0.63f * beside) > 3.f + u * (1.f / 55.f)) != 0;
}

// A tile, or a piece of one.
struct Unit {
  int row, begin, tokens, len;  // the row's first token in Q, how many, and its cached tokens
  int tile, part, parts;        // of the row; of the tile
  int tiles, first;             // the row's tiles and its first unit
};

// Up to 64 rows: a row to a lane, every wave for itself, with one load's wait and no
// barrier.  64 prompts of 128 tokens take 44 us, a prompt of 300 takes 17; 51 and 27 with
// the plan for any number of rows.
constexpr int kWaveRows = 64;
struct WavePlan {
  struct Shared {};
  int begin, tokens, len;
  RowWork w;
  int tile_end, unit_end;  // of this row, counted over the rows up to it
  int piece, units, tiles;

  __device__ __forceinline__ void make(const PrefillArgs& a, const Heads& heads, const Rows& rows, int room, int known, void*) {
    const int r = threadIdx.x & 63, group = heads.group.d, at = min(r, a.n_rows - 1);
    const int end = rows.cu_tokens[at + 1];
    begin = rows.cu_tokens[at];
    len = rows.seq_lens[at];
    w = work_of_row(a, group, begin, end, len);
    if (r >= a.n_rows || __any(end < begin)) w.tiles = 0;  // (descending offsets are none: rows may lie over each other)
    tokens = end - begin;
    tile_end = wave_scan(w.tiles, capped_add);
    tiles = __builtin_amdgcn_readlane(tile_end, 63);
    piece = known == 0 ? INT_MAX : known;
    if (known == 0 && tiles > 0 && tiles < room) {
      float blocks = (float)w.tiles * w.blocks, longest = w.tiles > 0 ? (float)w.blocks : 0.f;
      for (int m = 1; m < 64; m *= 2) {
        blocks += wave_xor_f(blocks, m);
        longest = fmaxf(longest, wave_xor_f(longest, m));
      }
      const Tries t = tries_of(tiles, blocks, room);
      piece = t.enough;
      for (int p0 = t.least; piece == t.enough && p0 < t.enough && p0 < t.least + 8; p0 += 4)
#pragma unroll
        for (int k = 3; k >= 0; --k) {
          const int n = wave_scan(w.tiles * pieces_of(w.blocks, p0 + k), capped_add);
          if (__builtin_amdgcn_readlane(n, 63) <= room) piece = p0 + k;
        }
      const int n = __builtin_amdgcn_readlane(wave_scan(w.tiles * pieces_of(w.blocks, piece), capped_add), 63);
      if (!worth(longest, piece, (int64_t)n * heads.n_kv.d)) piece = INT_MAX;
    }
    unit_end = wave_scan(w.tiles * pieces_of(w.blocks, piece), capped_add);
    units = __builtin_amdgcn_readlane(unit_end, 63);
  }
  // The row of unit (or of tile) x of the KV head.
  __device__ __forceinline__ Unit row_of(const Rows&, int x, bool is_tile) const {
    Unit n;
    n.row = (int)__builtin_ctzll(__ballot((is_tile ? tile_end : unit_end) > x));
    n.begin = __builtin_amdgcn_readlane(begin, n.row);
    n.tokens = __builtin_amdgcn_readlane(tokens, n.row);
    n.len = __builtin_amdgcn_readlane(len, n.row);
    n.tiles = __builtin_amdgcn_readlane(w.tiles, n.row);
    n.parts = pieces_of(__builtin_amdgcn_readlane(w.blocks, n.row), piece);
    n.first = __builtin_amdgcn_readlane(unit_end, n.row) - n.tiles * n.parts;
    n.part = 0;
    n.tile = is_tile ? x - (__builtin_amdgcn_readlane(tile_end, n.row) - n.tiles) : 0;
    return n;
  }
};

// Any number of rows: in LDS, a thread's rows one after another.
struct RowsPlan {
  struct Shared {
    int tiles[kMaxRows], blocks[kMaxRows], first_tile[kMaxRows + 1], first_unit[kMaxRows + 1], sums[4 * kWaves];
  };
  Shared* s;
  int piece, units, tiles;

  // The sum over the threads before this one, and over all.
  __device__ __forceinline__ int before(int mine, int* all) const {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, x = wave_scan(mine, capped_add);
    __syncthreads();  // (the last sums have been read)
    if (lane == 63) s->sums[wave] = x;
    __syncthreads();
    int sum = __builtin_amdgcn_update_dpp(0, x, 0x138, 0xf, 0xf, false);  // wave_shr 1
    *all = 0;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
      if (v == wave) sum = capped_add(sum, *all);
      *all = capped_add(*all, s->sums[v]);
    }
    *all = __builtin_amdgcn_readfirstlane(*all);
    return sum;
  }
  __device__ __forceinline__ void make(const PrefillArgs& a, const Heads& heads, const Rows& rows, int room, int known,
                                       void* shared) {
    s = static_cast<Shared*>(shared);
    const int t = threadIdx.x, group = heads.group.d;
    const int per = (a.n_rows + kThreads - 1) / kThreads;
    const int row0 = min(t * per, a.n_rows), row1 = min(row0 + per, a.n_rows);
    int mine = 0;
    float blocks = 0.f, longest = 0.f;
    bool descends = false;
    for (int r = row0; r < row1; ++r) {
      const int begin = rows.cu_tokens[r], end = rows.cu_tokens[r + 1];
      descends |= end < begin;
      const RowWork w = work_of_row(a, group, begin, end, rows.seq_lens[r]);
      s->tiles[r] = w.tiles;
      s->blocks[r] = w.blocks;
      mine = capped_add(mine, w.tiles);
      blocks += (float)w.tiles * w.blocks;
      if (w.tiles > 0) longest = fmaxf(longest, (float)w.blocks);
    }
    if (__syncthreads_or(descends)) {
      for (int r = row0; r < row1; ++r) s->tiles[r] = 0;
      mine = 0;
    }
    int sum = before(mine, &tiles);
    for (int r = row0; r < row1; ++r) {
      s->first_tile[r] = sum;
      sum = capped_add(sum, s->tiles[r]);
    }
    if (t == 0) s->first_tile[a.n_rows] = tiles;
    piece = known == 0 ? INT_MAX : known;
    if (known == 0 && tiles > 0 && tiles < room) {
      for (int m = 1; m < 64; m *= 2) {
        blocks += wave_xor_f(blocks, m);
        longest = fmaxf(longest, wave_xor_f(longest, m));
      }
      __syncthreads();
      if ((t & 63) == 0) {
        s->sums[t >> 6] = __float_as_int(blocks);
        s->sums[kWaves + (t >> 6)] = __float_as_int(longest);
      }
      __syncthreads();
      blocks = 0.f;
#pragma unroll
      for (int v = 0; v < kWaves; ++v) {
        blocks += __int_as_float(s->sums[v]);
        longest = fmaxf(longest, __int_as_float(s->sums[kWaves + v]));
      }
      const Tries tr = tries_of(tiles, blocks, room);
      piece = tr.enough;
      for (int p = tr.least; p < tr.enough && p < tr.least + 8; ++p) {
        int n = 0, all;
        for (int r = row0; r < row1; ++r) n = capped_add(n, s->tiles[r] * pieces_of(s->blocks[r], p));
        before(n, &all);
        if (all <= room) {
          piece = p;
          break;
        }
      }
      int n = 0, all;
      for (int r = row0; r < row1; ++r) n = capped_add(n, s->tiles[r] * pieces_of(s->blocks[r], piece));
      before(n, &all);
      if (!worth(longest, piece, (int64_t)all * heads.n_kv.d)) piece = INT_MAX;
    }
    mine = 0;
    for (int r = row0; r < row1; ++r) mine = capped_add(mine, s->tiles[r] * pieces_of(s->blocks[r], piece));
    sum = before(mine, &units);
    for (int r = row0; r < row1; ++r) {
      s->first_unit[r] = sum;
      sum = capped_add(sum, s->tiles[r] * pieces_of(s->blocks[r], piece));
    }
    if (t == 0) s->first_unit[a.n_rows] = units;
    __syncthreads();
    n_rows = a.n_rows;
  }
  int n_rows;
  __device__ __forceinline__ Unit row_of(const Rows& rows, int x, bool is_tile) const {
    Unit n;
    n.row = __builtin_amdgcn_readfirstlane(seq_of(is_tile ? s->first_tile : s->first_unit, n_rows, x));
    n.begin = rows.cu_tokens[n.row];
    n.tokens = rows.cu_tokens[n.row + 1] - n.begin;
    n.len = rows.seq_lens[n.row];
    n.tiles = __builtin_amdgcn_readfirstlane(s->tiles[n.row]);
    n.parts = pieces_of(__builtin_amdgcn_readfirstlane(s->blocks[n.row]), piece);
    n.first = __builtin_amdgcn_readfirstlane(s->first_unit[n.row]);
    n.part = 0;
    n.tile = is_tile ? x - __builtin_amdgcn_readfirstlane(s->first_tile[n.row]) : 0;
    return n;
  }
};

// Behind the parts: the blocks of a piece, for the join.
__device__ __forceinline__ int* piece_of_call(const PrefillArgs& a) {
  return reinterpret_cast<int*>(a.workspace + (size_t)kUnits * kPartFloats);
}

template <typename Plan>
__device__ __forceinline__ Unit unit_of(const Plan& plan, const Rows& rows, int u) {
  Unit n = plan.row_of(rows, u, false);
  const int local = u - n.first;
  n.part = n.parts == 1 ? 0 : __builtin_amdgcn_readfirstlane(local / max(n.tiles, 1));
  n.tile = n.tiles - 1 - (local - n.part * n.tiles);
  return n;
}

// Units are dealt out in bunches of neighbours, which read the same keys, to one XCD
// (workgroup j runs on XCD j % 8): bunch k of that XCD is bunch q = 8 k + x of all, of KV
// head q % H_kv.  Slot b of the launch gives KV head g and unit i of it (which may be
// past the last).
__device__ __forceinline__ void slot_of(int b, const Heads& heads, int units, int* g, int* i) {
  // (A bunch: 8, or where there are few units 4, 2 or 1, so that every XCD has some.  64
  // prompts of 128 tokens take 45 us, dealt out singly 48; long rows the same.)
  const int64_t all = (int64_t)units * heads.n_kv.d;
  const int shift = all >= 512 ? 3 : all >= 256 ? 2 : all >= 128 ? 1 : 0;
  const int x = b & 7, k = b >> 3;
  const int q = (k >> shift) * 8 + x, row = (int)heads.n_kv.of((uint32_t)q);
  *g = q - row * (int)heads.n_kv.d;
  *i = (row << shift) + (k & ((1 << shift) - 1));
}

template <int kFmt>
constexpr int kCodeBytes = kFmt == kCacheFp4 ? kHeadDim / 2 : kFmt == kCacheFp8 ? kHeadDim : 2 * kHeadDim;

// A row's keys in the cache.
struct Pages {
  const int32_t* table;  // the row's
  int n_pages, shift, last_key;
  int64_t page_bytes;
  uint32_t tok_bytes;
  // Byte offset of 16 keys from j0 (a multiple of 16) on, of the last ones where j0 is past them.
  __device__ __forceinline__ int64_t at(int j0) const {
    const int j = min(j0, last_key & ~15);
    const int page = min(max(table[j >> shift], 0), n_pages - 1);
    return page * page_bytes + (int64_t)(j & ((1 << shift) - 1)) * tok_bytes;
  }
};

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// x, of which the compiler knows nothing here: what is made of it is made where it is
// used, and not kept in registers over the steps.
template <typename T>
__device__ __forceinline__ T anew(T x) {
  asm volatile("" : "+v"(x));
  return x;
}
template <typename T>
__device__ __forceinline__ T anew_s(T x) {
  asm volatile("" : "+s"(x));
  return x;
}

// One tensor's block in registers on its way to LDS (FP8, FP4): of a wave 16 keys.
template <int kFmt>
struct Staged {
  static constexpr int kLoads = kFmt == kCacheFp8 ? 2 : 1;
  static constexpr int kRows = 16 / kLoads;  // of one load; 16 bytes to a lane
  uint4 codes[kLoads];
  uint32_t scale;
  // The wave's keys lie at `at`; past the row's last key, which is key `last` of them, that one again.
  __device__ __forceinline__ void load(const char* base, const char* scales, int64_t at, uint32_t tok_bytes, int last) {
    const int lane = threadIdx.x & 63, piece = lane % (64 / kRows);
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      const uint32_t r = (uint32_t)min(kRows * k + lane / (64 / kRows), last);
      codes[k] = *reinterpret_cast<const uint4*>(base + at + r * tok_bytes + 16u * piece);
      if (kFmt == kCacheFp4) scale = *reinterpret_cast<const uint8_t*>(scales + (at >> 4) + r * (tok_bytes >> 4) + piece);
    }
  }
  // Where the lane's pieces go in a block's rows: 256 row0 + (swz ^ ..), row0 16 run +
  // lane / .. (of the block's run of 16 keys) and the piece kPieces (lane % ..); the swizzle's bits that k and p give are
  // apart from the lane's.
  static constexpr int kPieces = kFmt == kCacheFp8 ? 2 : 4;  // of 16 bytes, of a load
  struct Place {
    uint32_t row, k_swz, v_swz;
  };
  static __device__ __forceinline__ Place place(int run) {
    const int lane = threadIdx.x & 63;
    const int row0 = 16 * run + lane / (64 / kRows), c0 = kPieces * (lane % (64 / kRows));
    return Place{256u * row0, 16u * (uint32_t)kswz(row0, c0), 16u * (uint32_t)vswz(row0, c0)};
  }
  // Piece p (of 4) of the lane's elements to the block at byte `lds` of LDS.
  __device__ __forceinline__ void store(const Place& to, uint32_t lds, bool is_v, int p) const {
    const int k = p / kPieces;
    const uint32_t bits = 16u * (p % kPieces) + (is_v ? 0u : 16u * kRows * k);
    const uint32_t at = anew(to.row + ((is_v ? to.v_swz : to.k_swz) ^ bits)) + lds + 256u * kRows * k;
    const uint32_t w[4] = {codes[k].x, codes[k].y, codes[k].z, codes[k].w};
    uint4 v;
    if constexpr (kFmt == kCacheFp8) {
      uint32_t x[4];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int z = (int)w[2 * (p % kPieces) + e];
        x[2 * e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(z, 1.f, false));
        x[2 * e + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(z, 1.f, true));
      }
      v = make_uint4(x[0], x[1], x[2], x[3]);
    } else {
      v = widen_e2m1(w[p], scale << 23);
    }
    *(__attribute__((address_space(3))) u32x4*)(uintptr_t)at = u32x4{v.x, v.y, v.z, v.w};
  }
};

template <int kFmt>
__device__ __forceinline__ float head_factor(const PrefillArgs& a, int head) {
  if (kFmt != kCacheFp8) return 1.f;
  const float m = a.cache.amax[head];
  return m > 0.f ? m / 448.f : 1.f;
}

// What a query's weighted values are multiplied by, of their sum l, with keys up to its last one (negative: none, and
// its result is 0).  Keys of no weight at all, from logits of -inf, give NaN.
__device__ __forceinline__ float result_factor(float factor, float l, int last) {
  return l > 0.f ? factor / l : last < 0 ? 0.f : __builtin_nanf("");
}

// Where query x of a row is in Q and O, and in lse.
__device__ __forceinline__ int64_t query_offset(const PrefillArgs& a, const Heads& heads, const Unit& n, int g, int x) {
  const int i = (int)heads.group.of(x), head = g * (int)heads.group.d + x - i * (int)heads.group.d;
  return head * a.q_head + (n.begin + i) * a.q_tok;
}
__device__ __forceinline__ int64_t query_lse(const PrefillArgs& a, const Heads& heads, const Unit& n, int g, int x) {
  const int i = (int)heads.group.of(x), head = g * (int)heads.group.d + x - i * (int)heads.group.d;
  return (int64_t)head * a.n_tokens + n.begin + i;
}

// The wave's 32 results, 64 elements of one in a lane, through 8 KB of LDS (pieces of
// 16 bytes swizzled by row) to whole rows: stored from the lanes as they are, in
// pieces of 8 bytes, 64 prompts of 128 tokens took 50 us and not 45.
__device__ __forceinline__ void write_queries(const PrefillArgs& a, const Heads& heads, const Unit& n, int g, int x0, int queries,
                                              const f32x16* o, float inv, unsigned char* lds) {
  const int lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int rq = 0; rq < 4; ++rq)
      *reinterpret_cast<uint2*>(lds + l32 * 256 + 16 * kswz(l32, 4 * dt + rq) + 8 * half) =
          make_uint2(two_bf16(o[dt][4 * rq] * inv, o[dt][4 * rq + 1] * inv),
                     two_bf16(o[dt][4 * rq + 2] * inv, o[dt][4 * rq + 3] * inv));
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int r = 4 * k + (lane >> 4), x = x0 + r;
    const uint4 w = *reinterpret_cast<const uint4*>(lds + r * 256 + 16 * kswz(r, lane & 15));
    if (x < queries) *reinterpret_cast<uint4*>(a.O + query_offset(a, heads, n, g, x) + 8 * (lane & 15)) = w;
  }
}

// The workgroup's LDS: two blocks of K and two of V, and
struct Tiles {
  unsigned char* k;
  unsigned char* v;
  int* bad;  // [kKeys]: the key's value is not finite
  float (*sums)[kWaves][32];  // maximum and sum of each wave's queries (attend_few)
};

__device__ __forceinline__ bool not_finite(uint32_t pair) {
  return (pair & 0x7f80u) == 0x7f80u || (pair & 0x7f800000u) == 0x7f800000u;
}

// A pair of values without those that are not finite.
__device__ __forceinline__ uint32_t finite_only(uint32_t z) {
  if ((z & 0x7f80u) == 0x7f80u) z &= 0xffff0000u;
  if ((z & 0x7f800000u) == 0x7f800000u) z &= 0xffffu;
  return z;
}

// The values of a key of the block at v that are not finite, added to the queries that attend it.
__device__ __forceinline__ void add_not_finite(const unsigned char* v, int key, int limit, int half, f32x16* o) {
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int rq = 0; rq < 4; ++rq) {
      const int d = 32 * dt + 8 * rq + 4 * half;
      const uint2 w = *reinterpret_cast<const uint2*>(v + key * 256 + 16 * vswz(key, d >> 3) + 2 * (d & 7));
      const float x[4] = {bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y)};
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (key <= limit && !(fabsf(x[e]) < INFINITY)) o[dt][4 * rq + e] += x[e];
    }
}

// Masked blocks: a weight of 0 times a value that is not finite would be NaN, so
// such values are taken out of the block and added to the queries that attend them.
// (Weights are positive, so the sum is the same whatever they are.)  limit: the
// lane's last key in the block.
__device__ __forceinline__ void take_out(unsigned char* v, int* bad, int limit, f32x16* o) {
  constexpr int kLoads = kBlockBytes / 16 / kThreads;
  const int tid = anew((int)threadIdx.x), half = (tid & 63) >> 5;
  bool any = false;
#pragma unroll
  for (int k = 0; k < kLoads; ++k) {
    const uint4 w = *reinterpret_cast<const uint4*>(v + 16 * (tid + kThreads * k));
    any |= not_finite(w.x) || not_finite(w.y) || not_finite(w.z) || not_finite(w.w);
  }
  if (!__syncthreads_or(any)) return;
  if (tid < kKeys) bad[tid] = 0;
  __syncthreads();
#pragma unroll 1
  for (int k = 0; k < kLoads; ++k) {
    const uint4 w = *reinterpret_cast<const uint4*>(v + 16 * (tid + kThreads * k));
    if (not_finite(w.x) || not_finite(w.y) || not_finite(w.z) || not_finite(w.w)) bad[(tid + kThreads * k) >> 4] = 1;
  }
  __syncthreads();
#pragma unroll 1
  for (int key = 0; key < kKeys; ++key) {
    if (__builtin_amdgcn_readfirstlane(bad[key]) == 0) continue;
    add_not_finite(v, key, limit, half, o);
  }
  __syncthreads();
#pragma unroll 1
  for (int k = 0; k < 4 * kLoads; ++k) {
    uint32_t* at = reinterpret_cast<uint32_t*>(v) + tid + kThreads * k;
    *at = finite_only(*at);
  }
  __syncthreads();
}

// The same of a wave's own 32 keys.
__device__ __forceinline__ void take_out_of_wave(unsigned char* v, int limit, f32x16* o) {
  const int lane = anew((int)threadIdx.x & 63);
  uint32_t bad = 0;  // a bit to a key
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const uint4 w = *reinterpret_cast<const uint4*>(v + 16 * (lane + 64 * k));
    const uint64_t any = __ballot(not_finite(w.x) || not_finite(w.y) || not_finite(w.z) || not_finite(w.w));
#pragma unroll
    for (int e = 0; e < 4; ++e) bad |= (any >> (16 * e) & 0xffff) != 0 ? 1u << (4 * k + e) : 0u;
  }
  if (bad == 0) return;
#pragma unroll 1
  for (uint32_t rest = bad; rest != 0; rest &= rest - 1) add_not_finite(v, __builtin_ctz(rest), limit, lane >> 5, o);
#pragma unroll 1
  for (int k = 0; k < 32; ++k) {
    uint32_t* at = reinterpret_cast<uint32_t*>(v) + lane + 64 * k;
    *at = finite_only(*at);
  }
  asm volatile("" ::: "memory");
}

// The order of instructions is that of the source here.
__device__ __forceinline__ void fence() { __builtin_amdgcn_sched_barrier(0); }

// One unit.  A step takes a block of 64 keys: the first product of the next block
// runs beside the exponentials of this one, and this one's second product beside
// the next one's maximum, an instruction of each in turn, so that the matrix core
// and the vector unit work at the same time.  One barrier to a step, at its start:
// the next K and this V are there, and the buffers of this K and the last V are free
// for the copies of the K after the next and the next V.
template <int kFmt, bool kLse>
__device__ __forceinline__ void attend_unit(const PrefillArgs& a, const Heads& heads, const Rows& rows, const Unit& n,
                                            int piece, int g, const Tiles& t, float* slot) {
  constexpr bool kCopied = kFmt == kCacheBf16;  // straight to LDS
  constexpr int kAhead = kCopied ? 4 : 3;       // operands on their way from LDS (no registers for a fourth beside the codes)
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, l32 = lane & 31;
  const int queries = n.tokens * (int)heads.group.d, x0 = n.tile * kQueries;
  const int64_t cap = (int64_t)a.max_pages << a.cache.page_shift;
  const int before = n.len - n.tokens;  // position of the row's first new token
  const int held = (int)min((int64_t)n.len, cap);
  const int tile_last = min(before + (int)heads.group.of(min(x0 + kQueries, queries) - 1), held - 1);

  Pages pages;
  pages.table = rows.page_table + (int64_t)n.row * a.max_pages;
  pages.n_pages = a.cache.n_pages;
  pages.shift = a.cache.page_shift;
  pages.last_key = max(tile_last, 0);
  pages.page_bytes = a.cache.page * kCodeBytes<kFmt> / kHeadDim;
  pages.tok_bytes = (uint32_t)(a.cache.tok * kCodeBytes<kFmt> / kHeadDim);
  const int blocks = tile_last < 0 ? 0 : tile_last / kKeys + 1;
  const int b0 = piece == INT_MAX ? 0 : n.part * piece;
  const int b1 = piece == INT_MAX ? blocks : min(blocks, b0 + piece);
  // The wave moves keys 16 wave .. + 15 of each block (all in one page).  Lane i holds
  // where those of block window + i are: a page number's load, waited for once in 64
  // blocks, would otherwise be one in every step.
  auto key0 = [&](int b) __attribute__((always_inline)) { return b * kKeys + 16 * wave; };
  int window = b0;
  int64_t places = pages.at(key0(min(b0 + lane, pages.last_key / kKeys)));
  auto place_of = [&](int b) __attribute__((always_inline)) {  // called with ascending b
    if (b >= window + 64) {
      window = b;
      places = pages.at(key0(min(b + lane, pages.last_key / kKeys)));
    }
    const int lo = __builtin_amdgcn_readlane((int)(uint32_t)places, b - window);
    const int hi = __builtin_amdgcn_readlane((int)(places >> 32), b - window);
    return (int64_t)((uint64_t)(uint32_t)hi << 32 | (uint32_t)lo);
  };

  const int first_last = min(before + (int)heads.group.of(x0), held - 1);  // the last key of the tile's first query
  const int plain = (first_last + 1) / kKeys;                               // blocks before it are attended whole
  // The lane's query (past the row's last one: that one, and not written).
  int last;  // its last key
  bf16x8 q[8];
  {
    const int x = min(x0 + 32 * wave + l32, queries - 1), i = (int)heads.group.of(x);
    last = min(before + i, held - 1);
    const uint16_t* row = a.Q + query_offset(a, heads, n, g, x) + 8 * half;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) q[ks] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(row + 16 * ks));
  }

  const int64_t head_bytes = g * a.cache.head * kCodeBytes<kFmt> / kHeadDim;
  const char* K = static_cast<const char*>(a.cache.K) + head_bytes;
  const char* V = static_cast<const char*>(a.cache.V) + head_bytes;
  const char* Ks = static_cast<const char*>(a.cache.K_scale) + g * a.cache.head / 32;
  const char* Vs = static_cast<const char*>(a.cache.V_scale) + g * a.cache.head / 32;
  const float scale_log2 = a.scale * kLog2e * head_factor<kFmt>(a, g);

  auto last_of = [&](int b) __attribute__((always_inline)) {  // the row's last key among them (15 if it is behind them)
    const int j = key0(b);
    return j > pages.last_key ? (pages.last_key & 15) : min(15, pages.last_key - j);
  };
  // BF16: four copies of four keys each, straight to LDS; copies c and c + 1.  Offset of
  // a lane in a run of 16 keys: row 4 c + lane / 16, piece lane % 16 as it is swizzled.
  uint32_t k_lds = __builtin_amdgcn_readfirstlane(lds_offset(t.k) + (uint32_t)wave * 4096u);
  uint32_t v_lds = __builtin_amdgcn_readfirstlane(lds_offset(t.v) + (uint32_t)wave * 4096u);
  const uint32_t row_off = (uint32_t)(lane >> 4) * pages.tok_bytes;
  const uint32_t k_piece = 16u * (uint32_t)kswz(lane >> 4, lane & 15), v_piece = 16u * (uint32_t)vswz(lane >> 4, lane & 15);
  auto copy = [&](bool is_v, int buf, int64_t at, int c0) __attribute__((always_inline)) {
    const char* run = (is_v ? V : K) + at;
    const uint32_t row_off_ = anew(row_off), tok_bytes = anew_s(pages.tok_bytes);
    const uint32_t lds = (is_v ? v_lds : k_lds) + (uint32_t)(buf * kBlockBytes);
#pragma unroll
    for (int c = c0; c < c0 + 2; ++c)
      lds_dma16(run + (size_t)(4 * c) * tok_bytes, row_off_ + (is_v ? v_piece : k_piece ^ (64u * c)), lds + 1024u * c);
  };
  // All four, where the row's last key may be among them or before them: past it, that one again.
  auto copy_last = [&](bool is_v, int buf, int64_t at, int b) __attribute__((always_inline)) {
    const char* run = (is_v ? V : K) + at;
    const uint32_t lds = (is_v ? v_lds : k_lds) + (uint32_t)(buf * kBlockBytes);
    const int top = last_of(b), l = anew(lane);
#pragma unroll 1
    for (int c = 0; c < 4; ++c) {
      const int r = 4 * c + (l >> 4), piece_at = is_v ? vswz(r, l & 15) : kswz(r, l & 15);
      lds_dma16(run, (uint32_t)min(r, top) * pages.tok_bytes + 16u * (uint32_t)piece_at, lds + 1024u * c);
    }
  };
  Staged<kCopied ? kCacheFp8 : kFmt> k_next, v_next;
  const uint32_t k_at0 = lds_offset(t.k), v_at0 = lds_offset(t.v);
  const typename Staged<kCopied ? kCacheFp8 : kFmt>::Place place = Staged<kCopied ? kCacheFp8 : kFmt>::place(wave);

  // Operands from LDS.  K: row 32 mt + l32, pieces 2 ks + half.  V (transposed): rows
  // 16 c + 4 half + (lane % 16) / 4 (and + 8), elements 32 dt + 16 ((lane / 16) % 2) + 4 (lane % 4).
  const int vq = (lane & 15) >> 2;
  uint32_t k_at[8], v_at[4];
  const uint32_t k_row = lds_offset(t.k) + (uint32_t)l32 * 256u, k_swz = 16u * (uint32_t)kswz(l32, half);
#pragma unroll
  for (int ks = 0; ks < 8; ++ks) k_at[ks] = k_row + (k_swz ^ (32u * ks));
  const uint32_t v_row = lds_offset(t.v) + (uint32_t)(4 * half + vq) * 256u + 8u * (lane & 1);
  const uint32_t v_swz = 16u * (uint32_t)vswz(vq, 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1));
#pragma unroll
  for (int dt = 0; dt < 4; ++dt) v_at[dt] = v_row + (v_swz ^ (64u * dt));
  typedef const __attribute__((address_space(3))) u32x4 lds_u32x4;
  auto k_frag = [&](int buf, int f) __attribute__((always_inline)) {  // f = 2 ks + mt, in this order
    return __builtin_bit_cast(bf16x8, *(lds_u32x4*)(uintptr_t)(k_at[f >> 1] + (uint32_t)(buf * kBlockBytes + (f & 1) * 8192)));
  };
  auto v_frag = [&](int buf, int f) __attribute__((always_inline)) {  // f = 4 c + dt
    const uint32_t at = v_at[f & 3] + (uint32_t)(buf * kBlockBytes + (f >> 2) * 4096);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)at);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)(at + 8 * 256));
    bf16x8 v;
    __builtin_memcpy(&v, &lo, 8);
    __builtin_memcpy(reinterpret_cast<unsigned char*>(&v) + 8, &hi, 8);
    return v;
  };

  float l = 0.f, l_exact = 0.f;  // this half wave's sums, of the weights as they are rounded and before it
  f32x16 o[4];
#pragma unroll
  for (int dt = 0; dt < 4; ++dt) o[dt] = f32x16{};
  float m = -INFINITY, shift = 0.f;  // the reference of the exponentials; shift: 0 where it is -inf

  auto mask = [&](f32x16* s, int b) __attribute__((always_inline)) {
    const int limit = anew(last) - b * kKeys;
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
      const int lim = limit - 32 * mt - 4 * half;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[mt][r] = (8 * (r >> 2) + (r & 3)) > lim ? -INFINITY : s[mt][r];
    }
  };
  auto top_of = [&](const f32x16* s) __attribute__((always_inline)) {
    float top = -INFINITY;
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, s[mt][r]);
    return top;
  };
  // The reference follows a maximum that exceeds it by much.  (Each query for itself:
  // its result does not depend on the wave's others.)
  auto follow = [&](float top) __attribute__((always_inline)) {
    const float m_new = top > m + kRescaleSlack ? top : m;
    const float f = m_new == m ? 1.f : fast_exp2(m - m_new);
    m = m_new;
    shift = m == -INFINITY ? 0.f : m;
    l *= f;
    l_exact *= f;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[dt][r] *= f;
  };

  constexpr int kLead = kCopied ? 2 : 3;  // blocks that the loads of K are ahead; those of V are one behind them
  int64_t at_v;                           // where the keys of the block whose V comes next are
  f32x16 s0[2], s1[2];
  uint32_t pw[16];  // the weights, pairs in bf16
  auto weigh = [&](int j, float e0, float e1) __attribute__((always_inline)) {  // pair j
    if (kLse) l_exact += e0 + e1;
    pw[j] = two_bf16(e0, e1);
    const uint32_t ones = 0x3f803f80u;
    l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pw[j]), __builtin_bit_cast(bf16x2, ones), l, false);
  };
  auto exponentials = [&](const f32x16* s, int j) __attribute__((always_inline)) {  // of pair j
    weigh(j, fast_exp2(fmaf(s[j >> 3][2 * (j & 7)], scale_log2, -shift)),
          fast_exp2(fmaf(s[j >> 3][2 * (j & 7) + 1], scale_log2, -shift)));
  };
  auto weights = [&](int c) __attribute__((always_inline)) {  // of 16 keys
    return __builtin_bit_cast(bf16x8, make_uint4(pw[4 * c], pw[4 * c + 1], pw[4 * c + 2], pw[4 * c + 3]));
  };
  auto logits = [&](int buf, f32x16* s) __attribute__((always_inline)) {
    bf16x8 f[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) f[k] = k_frag(buf, k);
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      fence();
      s[k & 1] = mfma_bf16(f[k % kAhead], q[k >> 1], k < 2 ? f32x16{} : s[k & 1]);
      if (k + kAhead < 16) f[k % kAhead] = k_frag(buf, k + kAhead);
    }
    fence();
  };
  // A step of block b, in buffers kBuf: its logits in s, the next block's to s_next.
  // For blocks attended whole that have at least four more behind them.
  auto step = [&](auto buf_of, int b, const f32x16* s, f32x16* s_next) __attribute__((always_inline)) {
    constexpr int kBuf = decltype(buf_of)::value;
    if constexpr (kCopied) RBS_WAIT_VMCNT(0);
    __syncthreads();
    asm volatile("" : "+s"(k_lds), "+s"(v_lds));  // (sums of these with constants are not kept from step to step)
    const int64_t at = at_v, at_k = place_of(b + kLead);
    at_v = at_k;
    // What goes to the free buffers, in four parts.
    auto move = [&](int part) __attribute__((always_inline)) {
      if constexpr (kCopied) {
        if (part < 2) copy(false, kBuf, at_k, 2 * part);
        else copy(true, kBuf ^ 1, at, 2 * (part - 2));
      } else if (part < 2) {
        k_next.store(place, k_at0 + kBuf * kBlockBytes, false, 2 * part);
        k_next.store(place, k_at0 + kBuf * kBlockBytes, false, 2 * part + 1);
        if (part == 1) k_next.load(K, Ks, at_k, pages.tok_bytes, 15);
      } else {
        v_next.store(place, v_at0 + (kBuf ^ 1) * kBlockBytes, true, 2 * (part - 2));
        v_next.store(place, v_at0 + (kBuf ^ 1) * kBlockBytes, true, 2 * (part - 2) + 1);
        if (part == 3) v_next.load(V, Vs, at, pages.tok_bytes, 15);
      }
    };
    // The exponentials in three stages, a stage of three pairs at a time: none waits for
    // the one before it.
    float arg[2], exp[2];
    auto stage = [&](int j) __attribute__((always_inline)) {
      if (j >= 2 && j < 18) weigh(j - 2, exp[0], exp[1]);
      if (j >= 1 && j < 17) {
        exp[0] = fast_exp2(arg[0]);
        exp[1] = fast_exp2(arg[1]);
      }
      if (j < 16) {
        arg[0] = fmaf(s[j >> 3][2 * (j & 7)], scale_log2, -shift);
        arg[1] = fmaf(s[j >> 3][2 * (j & 7) + 1], scale_log2, -shift);
      }
    };
    // First product of the next block; three quarters of the exponentials.
    bf16x8 f[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) f[k] = k_frag(kBuf ^ 1, k);
    fence();
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      s_next[k & 1] = mfma_bf16(f[k % kAhead], q[k >> 1], k < 2 ? f32x16{} : s_next[k & 1]);
      f[k % kAhead] = k + kAhead < 16 ? k_frag(kBuf ^ 1, k + kAhead) : v_frag(kBuf, k + kAhead - 16);
      if ((k & 3) != 3) stage(3 * (k >> 2) + (k & 3));
      else move(k >> 2);
      fence();
    }
    // Second product of this block; the last exponentials, and the next block's maximum.
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      o[k & 3] = mfma_bf16(f[(k + 16) % kAhead], weights(k >> 2), o[k & 3]);
      if (k + kAhead < 16) f[(k + 16) % kAhead] = v_frag(kBuf, k + kAhead);
      if (k < 6) stage(12 + k);
      else if (k >= 8)
#pragma unroll
        for (int e = 0; e < 4; ++e) top = fmaxf(top, s_next[(k >> 2) & 1][4 * (k & 3) + e]);
      fence();
    }
    top = half_max(top) * scale_log2;
    if (__any(top > m + kRescaleSlack)) follow(top);
  };
  // Any other block, in buffers buf: its logits in s0, then the next one's.
  auto step_of_any = [&](int buf, int b) __attribute__((always_inline)) {
    const bool more = b + 1 < b1, more2 = b + 2 < b1;
    if constexpr (kCopied) RBS_WAIT_VMCNT(0);
    __syncthreads();
    const int64_t at = at_v, at_k = place_of(b + kLead);
    at_v = at_k;
    if constexpr (kCopied) {
      if (more2) copy_last(false, buf, at_k, b + 2);
      if (more) copy_last(true, buf ^ 1, at, b + 1);
    } else {
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        if (more2) k_next.store(place, k_at0 + buf * kBlockBytes, false, p);
        if (more) v_next.store(place, v_at0 + (buf ^ 1) * kBlockBytes, true, p);
      }
      if (b + 3 < b1) k_next.load(K, Ks, at_k, pages.tok_bytes, last_of(b + 3));
      if (more2) v_next.load(V, Vs, at, pages.tok_bytes, last_of(b + 2));
    }
    if (b >= plain) take_out(t.v + buf * kBlockBytes, t.bad, last - b * kKeys, o);
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      exponentials(s0, j);
      if ((j & 3) == 3) fence();
    }
    if (more) logits(buf ^ 1, s0);
    bf16x8 f[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) f[k] = v_frag(buf, k);
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      fence();
      o[k & 3] = mfma_bf16(f[k % kAhead], weights(k >> 2), o[k & 3]);
      if (k + kAhead < 16) f[k % kAhead] = v_frag(buf, k + kAhead);
    }
    fence();
    if (!more) return;
    if (b + 1 >= plain) mask(s0, b + 1);
    const float top = half_max(top_of(s0)) * scale_log2;
    if (__any(top > m + kRescaleSlack)) follow(top);
  };

  if (b0 < b1) {
    const int64_t at = place_of(b0), at1 = place_of(b0 + 1);
    const bool two = b0 + 1 < b1;
    if constexpr (kCopied) {
      copy_last(false, 0, at, b0);
      copy_last(true, 0, at, b0);
      if (two) copy_last(false, 1, at1, b0 + 1);
      at_v = at1;
      RBS_WAIT_VMCNT(0);
    } else {
      k_next.load(K, Ks, at, pages.tok_bytes, last_of(b0));
      v_next.load(V, Vs, at, pages.tok_bytes, last_of(b0));
      Staged<kFmt> second;
      second.load(K, Ks, at1, pages.tok_bytes, last_of(b0 + 1));
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        k_next.store(place, k_at0, false, p);
        v_next.store(place, v_at0, true, p);
        second.store(place, k_at0 + kBlockBytes, false, p);
      }
      at_v = place_of(b0 + 2);
      if (b0 + 2 < b1) k_next.load(K, Ks, at_v, pages.tok_bytes, last_of(b0 + 2));
      if (two) v_next.load(V, Vs, at1, pages.tok_bytes, last_of(b0 + 1));
    }
    __syncthreads();
    logits(0, s0);
    if (b0 >= plain) mask(s0, b0);
    follow(half_max(top_of(s0)) * scale_log2);
    int b = b0;
    for (; b + 2 < plain && b + 5 < b1; b += 2) {
      step(std::integral_constant<int, 0>{}, b, s0, s1);
      step(std::integral_constant<int, 1>{}, b + 1, s1, s0);
    }
    for (int buf = 0; b < b1; ++b, buf ^= 1) step_of_any(buf, b);
  }

  if (x0 + 32 * wave >= queries) return;  // (no query of the wave's)
  l = half_sum(l);
  if (kLse) l_exact = half_sum(l_exact);
  if (n.parts == 1) {
    const float factor = head_factor<kFmt>(a, a.n_kv_heads + g);
    const float inv = result_factor(factor, l, last);
    const int x = x0 + 32 * wave + (anew(lane) & 31);
    if (kLse && half == 0 && x < queries)
      a.lse[query_lse(a, heads, n, g, x)] = l_exact == 0.f ? -INFINITY : (m + log2f(l_exact)) / kLog2e;
    // (K's buffers: every wave was done with them at the last step's barrier.)
    write_queries(a, heads, n, g, x0 + 32 * wave, queries, o, inv, t.k + 8192 * wave);
    return;
  }
  // A piece: every lane's 64 elements in runs of four, a KB for the wave at a time.
  if (b0 < b1) {
    float* out = slot + wave * 32 * kHeadDim;
    const int lane = anew((int)threadIdx.x) & 63;
#pragma unroll
    for (int k = 0; k < 16; ++k)
      *reinterpret_cast<float4*>(out + 4 * (64 * k + lane)) = make_float4(o[k >> 2][4 * (k & 3)], o[k >> 2][4 * (k & 3) + 1],
                                                                        o[k >> 2][4 * (k & 3) + 2], o[k >> 2][4 * (k & 3) + 3]);
  }
  if (half == 0) {
    float* sums = slot + kQueries * kHeadDim + 32 * wave + l32;
    sums[0] = m;
    sums[kQueries] = l;
    if (kLse) sums[2 * kQueries] = l_exact;
  }
}

// A unit of a row of at most 32 queries: a wave has all of them and every fourth block of
// 32 keys for itself, in its own quarter of LDS, so that no wave waits for another before
// the end, where the waves' sums are joined.  K of the wave's next block (FP8, FP4: its
// codes) is on its way during this one's exponentials and second product, V during the
// next first product.  32 rows of 4 tokens after 16000, 32 heads on 4, take 207 us in
// BF16, 129 in FP8 and 114 in FP4 on the GPU (5.1, 4.1 and 2.4 TB/s; FP4 is bound by the instructions of the
// widening and the softmax), with the weights in one part 207, 122 and 103; 218, 165 and 155 as tiles (with
// a costlier join); rows of 33 to 64 queries, two waves to a block, took 175 us in FP4 and as tiles 155.
template <int kFmt, bool kLse>
__device__ __forceinline__ void attend_few(const PrefillArgs& a, const Heads& heads, const Rows& rows, const Unit& n,
                                           int piece, int g, const Tiles& t, float* slot) {
  constexpr bool kCopied = kFmt == kCacheBf16;
  constexpr int kOwn = 32;  // keys of a block
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = lane >> 5, l32 = lane & 31;
  const int queries = n.tokens * (int)heads.group.d;
  const int before = n.len - n.tokens;
  const int held = (int)min((int64_t)n.len, (int64_t)a.max_pages << a.cache.page_shift);
  const int tile_last = min(before + n.tokens - 1, held - 1);

  Pages pages;
  pages.table = rows.page_table + (int64_t)n.row * a.max_pages;
  pages.n_pages = a.cache.n_pages;
  pages.shift = a.cache.page_shift;
  pages.last_key = max(tile_last, 0);
  pages.page_bytes = a.cache.page * kCodeBytes<kFmt> / kHeadDim;
  pages.tok_bytes = (uint32_t)(a.cache.tok * kCodeBytes<kFmt> / kHeadDim);
  const int last_block = pages.last_key / kOwn, blocks = tile_last < 0 ? 0 : last_block + 1;
  constexpr int kPer = kKeys / kOwn;
  const int b0 = (piece == INT_MAX ? 0 : n.part * piece * kPer) + wave;
  const int b1 = piece == INT_MAX ? blocks : min(blocks, (n.part + 1) * piece * kPer);
  // Lane i holds where run i % 2 (of 16 keys) of the wave's block window + i / 2 is.
  int window = b0;
  auto look = [&](int b) __attribute__((always_inline)) {
    return pages.at(min(b + kWaves * (lane >> 1), last_block) * kOwn + 16 * (lane & 1));
  };
  int64_t places = look(b0);
  auto place_of = [&](int b, int run) __attribute__((always_inline)) {  // called with ascending b
    if (b >= window + 32 * kWaves) {
      window = b;
      places = look(b);
    }
    const int i = 2 * ((b - window) / kWaves) + run;
    const int lo = __builtin_amdgcn_readlane((int)(uint32_t)places, i);
    const int hi = __builtin_amdgcn_readlane((int)(places >> 32), i);
    return (int64_t)((uint64_t)(uint32_t)hi << 32 | (uint32_t)lo);
  };
  auto last_of = [&](int b, int run) __attribute__((always_inline)) {  // the row's last key among the run's (15 if it is behind them)
    const int left = pages.last_key - b * kOwn - 16 * run;
    return left < 0 ? pages.last_key & 15 : min(15, left);
  };
  const int first_last = min(before, held - 1);   // the last key of the row's first query
  const int plain = (first_last + 1) / kOwn;      // blocks before it are attended whole
  int last;
  bf16x8 q[8];
  {
    const int x = min(l32, queries - 1), i = (int)heads.group.of(x);
    last = min(before + i, held - 1);
    const uint16_t* row = a.Q + query_offset(a, heads, n, g, x) + 8 * half;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) q[ks] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(row + 16 * ks));
  }
  const int64_t head_bytes = g * a.cache.head * kCodeBytes<kFmt> / kHeadDim;
  const char* K = static_cast<const char*>(a.cache.K) + head_bytes;
  const char* V = static_cast<const char*>(a.cache.V) + head_bytes;
  const char* Ks = static_cast<const char*>(a.cache.K_scale) + g * a.cache.head / 32;
  const char* Vs = static_cast<const char*>(a.cache.V_scale) + g * a.cache.head / 32;
  const float scale_log2 = a.scale * kLog2e * head_factor<kFmt>(a, g);

  // The wave's LDS: K, then V.
  unsigned char* own = t.k + wave * 2 * kOwn * 256;
  const uint32_t k_lds = __builtin_amdgcn_readfirstlane(lds_offset(own)), v_lds = k_lds + kOwn * 256;
  auto copy = [&](bool is_v, int b) __attribute__((always_inline)) {
#pragma unroll
    for (int run = 0; run < 2; ++run) {
      const char* from = (is_v ? V : K) + place_of(b, run);
      const int top = last_of(b, run);
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int r = 4 * c + (lane >> 4), piece_at = is_v ? vswz(r, lane & 15) : kswz(r, lane & 15);
        lds_dma16(from, (uint32_t)min(r, top) * pages.tok_bytes + 16u * (uint32_t)piece_at,
                  (is_v ? v_lds : k_lds) + 4096u * run + 1024u * c);
      }
    }
  };
  typedef Staged<kCopied ? kCacheFp8 : kFmt> Codes;
  Codes k_next[2], v_next[2];
  const typename Codes::Place place = Codes::place(0);
  auto load = [&](Codes* to, bool is_v, int b) __attribute__((always_inline)) {
#pragma unroll
    for (int run = 0; run < 2; ++run)
      to[run].load(is_v ? V : K, is_v ? Vs : Ks, place_of(b, run), pages.tok_bytes, last_of(b, run));
  };
  auto widen = [&](const Codes* from, bool is_v) __attribute__((always_inline)) {
#pragma unroll
    for (int run = 0; run < 2; ++run)
#pragma unroll
      for (int p = 0; p < 4; ++p) from[run].store(place, (is_v ? v_lds : k_lds) + 4096u * run, is_v, p);
  };

  const int vq = (lane & 15) >> 2;
  const uint32_t k_row = k_lds + (uint32_t)l32 * 256u, k_swz = 16u * (uint32_t)kswz(l32, half);
  const uint32_t v_row = v_lds + (uint32_t)(4 * half + vq) * 256u + 8u * (lane & 1);
  const uint32_t v_swz = 16u * (uint32_t)vswz(vq, 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1));
  typedef const __attribute__((address_space(3))) u32x4 lds_u32x4;

  float l = 0.f, m = -INFINITY, shift = 0.f;
  f32x16 o[4];
#pragma unroll
  for (int dt = 0; dt < 4; ++dt) o[dt] = f32x16{};

  if (b0 < b1) {
    if constexpr (kCopied) {
      copy(false, b0);
      copy(true, b0);
    } else {
      load(k_next, false, b0);
      load(v_next, true, b0);
    }
  }
#pragma unroll 1
  for (int b = b0; b < b1; b += kWaves) {
    const int next = b + kWaves;
    const bool more = next < b1;
    if constexpr (kCopied) RBS_WAIT_VMCNT(8);  // (the eight copies of V may be on their way)
    else widen(k_next, false);
    f32x16 s{};
    const uint32_t k_swz_ = anew(k_swz);
    asm volatile("" ::: "memory");
#pragma unroll
    for (int ks = 0; ks < 8; ++ks)
      s = mfma_bf16(__builtin_bit_cast(bf16x8, *(lds_u32x4*)(uintptr_t)(k_row + (k_swz_ ^ (32u * ks)))), q[ks], s);
    if (more) {
      if constexpr (kCopied) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // K has been read
        copy(false, next);
      } else {
        load(k_next, false, next);
      }
    }
    fence();
    if (b >= plain) {
      const int lim = last - b * kOwn - 4 * half;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = (8 * (r >> 2) + (r & 3)) > lim ? -INFINITY : s[r];
    }
    float top = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) top = fmaxf(top, s[r]);
    top = half_max(top) * scale_log2;
    if (__any(top > m + kRescaleSlack)) {
      const float m_new = top > m + kRescaleSlack ? top : m;
      const float f = m_new == m ? 1.f : fast_exp2(m - m_new);
      m = m_new;
      shift = m == -INFINITY ? 0.f : m;
      l *= f;
#pragma unroll
      for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] *= f;
    }
    // Two bf16 parts: the weight cut off, and the rest, off by 2^-16 of the weight together.  The
    // rest is taken of the weight and 2^-22 of it: as positive as the weight is, so that
    // an infinite value stays one (with 0, or a rest below 0, it would be NaN).
    uint32_t pw[8], rest[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float e0 = fast_exp2(fmaf(s[2 * j], scale_log2, -shift)), e1 = fast_exp2(fmaf(s[2 * j + 1], scale_log2, -shift));
      l += e0 + e1;
      pw[j] = __builtin_amdgcn_perm(__float_as_uint(e1), __float_as_uint(e0), 0x07060302u);
      constexpr float kAbove = 1.f + 1.f / (1 << 22);
      rest[j] = two_bf16(fmaf(e0, kAbove, -bf16_lo(pw[j])), fmaf(e1, kAbove, -bf16_hi(pw[j])));
    }
    if constexpr (kCopied) {
      if (more) RBS_WAIT_VMCNT(8);  // (the next K's copies)
      else RBS_WAIT_VMCNT(0);
    } else {
      widen(v_next, true);
    }
    asm volatile("" ::: "memory");
    if (b >= plain) take_out_of_wave(own + kOwn * 256, last - b * kOwn, o);
    const uint32_t v_swz_ = anew(v_swz);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      fence();
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) {
        const uint32_t at = v_row + (v_swz_ ^ (64u * dt)) + 4096u * c;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)at);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)(at + 8 * 256));
        bf16x8 v;
        __builtin_memcpy(&v, &lo, 8);
        __builtin_memcpy(reinterpret_cast<unsigned char*>(&v) + 8, &hi, 8);
        o[dt] = mfma_bf16(v, __builtin_bit_cast(bf16x8, make_uint4(pw[4 * c], pw[4 * c + 1], pw[4 * c + 2], pw[4 * c + 3])), o[dt]);
        o[dt] = mfma_bf16(v, __builtin_bit_cast(bf16x8, make_uint4(rest[4 * c], rest[4 * c + 1], rest[4 * c + 2], rest[4 * c + 3])), o[dt]);
      }
    }
    fence();
    if (more) {
      if constexpr (kCopied) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // V has been read
        copy(true, next);
      } else {
        load(v_next, true, next);
      }
    }
  }

  // The waves' sums, joined: each takes a quarter of the elements from all of them.
  l = half_sum(l);
  asm volatile("" ::: "memory");
#pragma unroll
  for (int k = 0; k < 16; ++k)
    *reinterpret_cast<float4*>(own + 16 * (64 * k + lane)) = make_float4(o[k >> 2][4 * (k & 3)], o[k >> 2][4 * (k & 3) + 1],
                                                                         o[k >> 2][4 * (k & 3) + 2], o[k >> 2][4 * (k & 3) + 3]);
  if (half == 0) {
    t.sums[0][wave][l32] = m;
    t.sums[1][wave][l32] = l;
  }
  __syncthreads();
  float top = t.sums[0][0][l32];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) top = fmaxf(top, t.sums[0][w][l32]);
  const float ref = top == -INFINITY ? 0.f : top;
  float f[kWaves];
  l = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {  // (a wave without keys: a factor of 0, sums of 0; a NaN stays one under any factor)
    f[w] = fast_exp2(t.sums[0][w][l32] - ref);
    l += t.sums[1][w][l32] * f[w];
  }
  const bool whole = n.parts == 1, mine = l32 < queries;
  const float factor = head_factor<kFmt>(a, a.n_kv_heads + g);
  const float inv = result_factor(factor, l, last);
  if (half == 0 && wave == 0) {
    if (!whole) {
      float* sums = slot + kQueries * kHeadDim + l32;
      sums[0] = top;
      sums[kQueries] = l;
      if (kLse) sums[2 * kQueries] = l;
    } else if (kLse && mine) {
      a.lse[query_lse(a, heads, n, g, l32)] = l == 0.f ? -INFINITY : (top + log2f(l)) / kLog2e;
    }
  }
  uint16_t* out = a.O + query_offset(a, heads, n, g, min(l32, queries - 1)) + 4 * half;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int k = 4 * wave + e;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float4 p = *reinterpret_cast<const float4*>(t.k + w * 2 * kOwn * 256 + 16 * (64 * k + lane));
      v.x += p.x * f[w]; v.y += p.y * f[w]; v.z += p.z * f[w]; v.w += p.w * f[w];
    }
    if (!whole) *reinterpret_cast<float4*>(slot + 4 * (64 * k + lane)) = v;
    else if (mine) *reinterpret_cast<uint2*>(out + 8 * k) = make_uint2(two_bf16(v.x * inv, v.y * inv), two_bf16(v.z * inv, v.w * inv));
  }
}

template <int kFmt, bool kLse, typename Plan>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void paged_prefill_kernel(PrefillArgs a,
                                                                                                         Heads heads,
                                                                                                         int room,
                                                                                                         RBS_ROWS_ARGS) {
  const Rows rows{page_table, seq_lens, cu_tokens};
  __shared__ __align__(1024) unsigned char tiles[4 * kBlockBytes + 128];
  __shared__ int bad[kKeys];
  __shared__ float sums[2][kWaves][32];
  const Tiles t{tiles, tiles + 2 * kBlockBytes, bad, sums};
  static_assert(sizeof(RowsPlan::Shared) <= sizeof(tiles), "the plan lies where the tiles will be");
  Plan plan;
  plan.make(a, heads, rows, room, 0, tiles);
  if (room > 0 && blockIdx.x == 0 && threadIdx.x == 0) *piece_of_call(a) = plan.piece;
  int g, i;
  slot_of(blockIdx.x, heads, plan.units, &g, &i);
  if (i >= plan.units) return;
  const Unit n = unit_of(plan, rows, i);
  if (std::is_same<Plan, RowsPlan>::value) __syncthreads();  // every wave has read the plan
  float* slot = n.parts > 1 ? a.workspace + (size_t)(g * plan.units + i) * kPartFloats : nullptr;
  if (n.tokens * (int)heads.group.d <= kFewQueries) attend_few<kFmt, kLse>(a, heads, rows, n, plan.piece, g, t, slot);
  else attend_unit<kFmt, kLse>(a, heads, rows, n, plan.piece, g, t, slot);
}

// Joins the pieces of a tile, in their order: an item is 32 queries and 32 of their
// elements, a wave takes every fourth piece.  Bound by latency: the loads of kBatch pieces
// of a wave are on their way together.  At most kJoiners workgroups, which make the plan
// once for all their items, and not at all where the tiles are whole: with a workgroup to
// an item, 256 tokens of 4 rows after 1024 each took 63 us and not 34.
template <typename Plan>
constexpr int kJoiners = std::is_same<Plan, WavePlan>::value ? 1024 : 256;  // (as many as fit at once)
template <int kFmt, typename Plan, typename Part>
__device__ __forceinline__ void join_item(const PrefillArgs& a, const Heads& heads, const Rows& rows, const Plan& plan,
                                          int item, Part& part) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = lane >> 5, l32 = lane & 31;
  const int all = plan.tiles * a.n_kv_heads, y = __builtin_amdgcn_readfirstlane(item / all), x = item - y * all;
  const int tile = (int)heads.n_kv.of((uint32_t)x), g = x - tile * a.n_kv_heads;
  const int dt = y & 3, q0 = 32 * (y >> 2);
  const Unit n = plan.row_of(rows, tile, true);
  const int queries = n.tokens * (int)heads.group.d, x0 = n.tile * kQueries + q0;
  if (n.parts == 1 || x0 >= queries) return;
  __syncthreads();  // (the last item has been read)
  // The pieces behind the tile's last block wrote no values.
  const int64_t cap = (int64_t)a.max_pages << a.cache.page_shift;
  const int last_query = min((n.tile + 1) * kQueries, queries) - 1;
  const int before = n.len - n.tokens, held = (int)min((int64_t)n.len, cap);
  const int tile_last = min(before + (int)heads.group.of(last_query), held - 1);
  const int parts = tile_last < 0 ? 0 : min(n.parts, pieces_of(tile_last / kKeys + 1, plan.piece));
  const float* slots = a.workspace + (size_t)(g * plan.units + n.first + n.tiles - 1 - n.tile) * kPartFloats;
  const size_t step = (size_t)n.tiles * kPartFloats;
  const int at = kQueries * kHeadDim + q0 + l32;
  float m = -INFINITY, l = 0.f, l_exact = 0.f;
  float4 o[4] = {};
  constexpr int kBatch = 4;
  for (int p0 = wave; p0 < parts; p0 += kWaves * kBatch) {
    float pm[kBatch], pl[kBatch], pe[kBatch];
    float4 w[kBatch][4];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const float* slot = slots + min(p0 + kWaves * k, parts - 1) * step;
      pm[k] = slot[at];
      pl[k] = slot[at + kQueries];
      pe[k] = a.lse != nullptr ? slot[at + 2 * kQueries] : 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        w[k][e] = *reinterpret_cast<const float4*>(slot + q0 * kHeadDim + 4 * (64 * (4 * dt + e) + lane));
    }
    float top = m;
#pragma unroll
    for (int k = 0; k < kBatch; ++k) top = fmaxf(top, pm[k]);
    const float ref = top == -INFINITY ? 0.f : top, keep = fast_exp2(m - ref);
    m = top;
    l *= keep;
    l_exact *= keep;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      o[e].x *= keep; o[e].y *= keep; o[e].z *= keep; o[e].w *= keep;
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      if (p0 + kWaves * k >= parts) continue;
      const float f = fast_exp2(pm[k] - ref);
      l += pl[k] * f;
      l_exact += pe[k] * f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        o[e].x += w[k][e].x * f; o[e].y += w[k][e].y * f; o[e].z += w[k][e].z * f; o[e].w += w[k][e].w * f;
      }
    }
  }
  if (half == 0) {
    part.m[wave][l32] = m;
    part.l[wave][l32] = l;
    part.l_exact[wave][l32] = l_exact;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) part.o[wave][e][lane] = o[e];
  __syncthreads();
  // Each wave joins a quarter of the elements.
  float top = part.m[0][l32];
#pragma unroll
  for (int v = 1; v < kWaves; ++v) top = fmaxf(top, part.m[v][l32]);
  const float ref = top == -INFINITY ? 0.f : top;
  l = l_exact = 0.f;
  float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int v = 0; v < kWaves; ++v) {
    const float f = fast_exp2(part.m[v][l32] - ref);
    l += part.l[v][l32] * f;
    l_exact += part.l_exact[v][l32] * f;
    const float4 w = part.o[v][wave][lane];
    r.x += w.x * f; r.y += w.y * f; r.z += w.z * f; r.w += w.w * f;
  }
  const int mine = x0 + l32;
  if (mine >= queries) return;
  const int last = min(before + (int)heads.group.of(mine), held - 1);
  const float inv = result_factor(head_factor<kFmt>(a, a.n_kv_heads + g), l, last);
  *reinterpret_cast<uint2*>(a.O + query_offset(a, heads, n, g, mine) + 32 * dt + 8 * wave + 4 * half) =
      make_uint2(two_bf16(r.x * inv, r.y * inv), two_bf16(r.z * inv, r.w * inv));
  if (a.lse != nullptr && half == 0 && dt == 0 && wave == 0)
    a.lse[query_lse(a, heads, n, g, mine)] = l_exact == 0.f ? -INFINITY : (top + log2f(l_exact)) / kLog2e;
}

template <int kFmt, typename Plan>
__global__ __launch_bounds__(kThreads) void paged_prefill_join_kernel(PrefillArgs a, Heads heads, RBS_ROWS_ARGS) {
  const Rows rows{page_table, seq_lens, cu_tokens};
  __shared__ typename Plan::Shared plan_lds;
  __shared__ struct {
    float m[kWaves][32], l[kWaves][32], l_exact[kWaves][32];
    float4 o[kWaves][4][64];
  } part;
  const int piece = __builtin_amdgcn_readfirstlane(*piece_of_call(a));
  if (piece == INT_MAX) return;
  Plan plan;
  plan.make(a, heads, rows, 0, piece, &plan_lds);
  const int items = 16 * plan.tiles * a.n_kv_heads;
  for (int item = blockIdx.x; item < items; item += gridDim.x) join_item<kFmt>(a, heads, rows, plan, item, part);
}

template <int kFmt>
hipError_t launch(const PrefillArgs& a, hipStream_t s) {
  const int group = a.n_q_heads / a.n_kv_heads;
  // At most so many tiles of a KV head.
  const int64_t tiles = (int64_t)a.n_tokens * group / kQueries + (a.n_rows < a.n_tokens ? a.n_rows : a.n_tokens);
  const int64_t keys = (int64_t)a.max_pages << a.cache.page_shift;  // of a row, at most
  const int64_t units = tiles * a.n_kv_heads;
  const bool split = units < kUnits && keys > kLeast * kKeys;
  const int room = split ? kUnits / a.n_kv_heads : 0;
  // (Bunches round up a head's units, and the XCDs' shares of them.)
  const int grid = (int)((split ? kUnits : units) + 64 + 8 * a.n_kv_heads);
  const Heads heads{Divisor((uint32_t)group), Divisor((uint32_t)a.n_kv_heads)};
  const bool few = a.n_rows <= kWaveRows;
  const auto kernel = few ? (a.lse != nullptr ? paged_prefill_kernel<kFmt, true, WavePlan> : paged_prefill_kernel<kFmt, false, WavePlan>)
                          : (a.lse != nullptr ? paged_prefill_kernel<kFmt, true, RowsPlan> : paged_prefill_kernel<kFmt, false, RowsPlan>);
  hipLaunchKernelGGL(kernel, dim3(grid), dim3(kThreads), 0, s, a, heads, room, a.page_table, a.seq_lens, a.cu_tokens);
  if (split) {
    const auto join = few ? paged_prefill_join_kernel<kFmt, WavePlan> : paged_prefill_join_kernel<kFmt, RowsPlan>;
    const int items = 16 * (int)units, most = few ? kJoiners<WavePlan> : kJoiners<RowsPlan>;
    hipLaunchKernelGGL(join, dim3(items < most ? items : most), dim3(kThreads), 0, s, a, heads, a.page_table, a.seq_lens,
                       a.cu_tokens);
  }
  return hipGetLastError();
}

}  // namespace

size_t prefill_workspace_bytes() { return sizeof(float) * (kUnits * kPartFloats + 4); }

hipError_t launch_paged_prefill(const PrefillArgs& a, hipStream_t s) {
  switch (a.cache.format) {
    case kCacheBf16: return launch<kCacheBf16>(a, s);
    case kCacheFp8: return launch<kCacheFp8>(a, s);
    case kCacheFp4: return launch<kCacheFp4>(a, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace rbs
