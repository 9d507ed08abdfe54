// The paged cache: where a tile's codes and parameters lie, and the launchers' arguments.  (perf/operators.py lays pools out by
// this description; a change of it is a change there.)
//
// A tile is 64 rows of one unit.  Its bytes, in this order: key codes, value codes, key parameters, value parameters (the
// last two only with codes).  Codes come in units of eight -- eight kept channels of one row for keys, eight rows of one
// channel for values -- which is what one lane hands to a 16x16x32 matrix instruction as its share of an operand, so that a
// lane's loads are its operands and no data crosses lanes or LDS between memory and the matrix cores.  64 units form a group:
//   keys:   group c = channels 8 c .. 8 c + 7; its unit (j, m) is row 16 j + m;
//   values: group (g, h, half) = rows {32 g + 16 x + 4 h + r}, element 4 x + r of a unit; its unit (j, m) is channel
//           64 half + 4 m + j.  (The rows are those whose logits a lane of quarter h holds after the first product.)
// Inside a group the units lie so that lane m finds its four (j = 0..3) in 16-byte cells that are contiguous over the 16
// lanes: cell k of lane m is at (16 k + m) * 16.
//   unit of 4 bytes (4-bit codes):  cell 0 = j 0..3
//   unit of 8 bytes (8-bit codes):  cell k = j 2 k, 2 k + 1
//   unit of 16 bytes (bf16):        cell k = j k
//   unit of 32 bytes (fp32):        cells 2 j, 2 j + 1
// 4-bit units hold code 2 p at bits 4 p and code 2 p + 1 at bits 16 + 4 p: two neighbours are one shift and one mask away
// from the two halves of a word.
// A parameter is a pair (scale, minimum) of the element type; the pairs of a group's eight channels (keys) or rows (values)
// lie together, groups in order.
#pragma once
#include "thk_internal.h"

namespace thk {

constexpr int kTile = 64;          // rows of a tile
constexpr int kValueGroups = 16;   // groups of a tile's values: 2 x 4 row octets, 2 halves of the channels

struct PagedLayout {
  int32_t chunks;      // groups of a tile's keys: T / 8, rounded up
  int32_t unit_bytes;
  int32_t v_codes;     // byte offsets from the tile's start
  int32_t k_params, v_params;
  int32_t tile_bytes;
};
constexpr PagedLayout paged_layout(int dtype, int bits, int T) {
  const int e = dtype == THK_BF16 ? 2 : 4;
  PagedLayout p{};
  p.chunks = (T + 7) / 8;
  p.unit_bytes = bits != 0 ? bits : 8 * e;
  p.v_codes = p.chunks * 64 * p.unit_bytes;
  p.k_params = p.v_codes + kValueGroups * 64 * p.unit_bytes;
  p.v_params = p.k_params + (bits != 0 ? p.chunks * 8 * 2 * e : 0);
  p.tile_bytes = p.v_params + (bits != 0 ? kValueGroups * 8 * 2 * e : 0);
  return p;
}
constexpr int kMostTileBytes = 65536;   // fp32 elements, all channels
constexpr int kMostTilesOfPage = 65536 / kTile;
static_assert(paged_layout(THK_F32, 0, kD).tile_bytes == kMostTileBytes && paged_layout(THK_F32, 8, kD).tile_bytes < kMostTileBytes);
static_assert((int64_t)kMostTileBytes * kMostTilesOfPage <= INT32_MAX);   // offsets inside a head's part of a page are 32-bit numbers

// An element that is the same for all lanes and that no kernel of the call writes, through the scalar cache: it does not wait
// for vector loads that are under way.
__device__ __forceinline__ int scalar_load(const int32_t *p, int64_t i) {
  return ((__attribute__((address_space(4))) const int32_t *)(uintptr_t)p)[i];
}

// Division by a number that is known when the call is planned, as a product: n * ceil(2^s / d) >> s is n / d for n < 2^24,
// with s = 40 for d < 2^16 (the rounding up adds less than n / 2^40 < 2^-16 < 1 / d) and 48 from there on (the product stays
// below 2^64 in both).  A division costs a wave some 30 instructions in front of its first load.
struct Divisor {
  uint64_t inv;
  int32_t shift;
  explicit Divisor(int64_t d = 1) : inv((((uint64_t)1 << (d < 65536 ? 40 : 48)) + d - 1) / d), shift(d < 65536 ? 40 : 48) {}
  __device__ __forceinline__ uint32_t of(uint32_t n) const { return (uint32_t)((n * inv) >> shift); }
};

// A block's place among layers, sequences and KV heads.
struct UnitPlace { uint32_t l; int b, h; };

// One unit's pages: the same for all lanes.
struct UnitPages {
  char *base;             // of the unit's part of page 0
  int64_t stride;         // from page to page
  const int32_t *row;     // the sequence's row of the table
  uint32_t n_pages;
  int32_t max_pages, tpp_shift, tile_bytes;

  // The table's entry for tile t of the sequence (for tiles past the table's end the last one), and the tile in that page;
  // nullptr where the page is none of the pool's.  t < 2^31 / 64 + a step.
  __device__ __forceinline__ int page_of(int t) const { return scalar_load(row, min(t >> tpp_shift, max_pages - 1)); }
  __device__ __forceinline__ char *in_page(int page, int t) const {
    if ((uint32_t)page >= n_pages) return nullptr;   // (negative ones among them)
    return base + page * stride + (uint32_t)(t & ((1 << tpp_shift) - 1)) * (uint32_t)tile_bytes;
  }
  __device__ __forceinline__ char *tile(int64_t t) const {
    if (t >> tpp_shift >= max_pages) return nullptr;
    return in_page(page_of((int)t), (int)t);
  }
};

// The pool and the tables of a call.
struct PagedPool {
  void *pool;
  const int32_t *table;    // [B][max_pages]
  int64_t n_pages;         // pages of one layer's part of the pool, < 2^31
  int32_t max_pages;
  int32_t tpp_shift;       // log2 of the tiles of a page
  int32_t N_kv, B;
  Divisor by_N_kv, by_B;
  PagedLayout lay;

  __device__ __forceinline__ UnitPlace place(uint32_t u) const {
    const uint32_t lb = by_N_kv.of(u), l = by_B.of(lb);
    return {l, (int)(lb - l * (uint32_t)B), (int)(u - lb * (uint32_t)N_kv)};
  }
  __device__ __forceinline__ UnitPages unit(const UnitPlace &w) const {
    const int64_t part = (int64_t)lay.tile_bytes << tpp_shift;   // a KV head's part of a page (at most 64 MB)
    return {(char *)pool + ((int64_t)w.l * n_pages * N_kv + w.h) * part, part * N_kv, table + (int64_t)w.b * max_pages,
            (uint32_t)n_pages, max_pages, tpp_shift, lay.tile_bytes};
  }
};

struct PagedWriteArgs {
  PagedPool p;
  const void *k, *v;
  const int16_t *idx;
  const int32_t *n_rows, *row0;   // [B]; row0 may be nullptr (0)
  int64_t src_rows;               // rows per unit of k and v
  int64_t most;                   // most rows of a sequence in this call
  int64_t units;
  int32_t T, tiles;               // tiles: blocks per unit, those of `most` rows
  Divisor by_tiles;
  bool apart;                     // keys and values by blocks of their own
};
// Keys and values of a tile by blocks of their own: where these are on the card all at once, eight (bf16) or four (fp32, by their
// LDS) on a compute unit.  Each then has half the work.  (One rule for writes and reads: bf16 reads of 1024 tiles lose 6 % by it, writes
// gain 15 %.)  One block or two, in us: bf16 4 bits, 512 tiles written in 7.7 or 6.9,
// read in 8.0 or 6.8; 1024: 12.2 or 10.4, 11.4 or 12.1; 2048: 21.6 or 21.1, 18.1 or 19.2; 16384: 108 or 138, 92 or 100.  fp32 8 bits,
// 384: 10.9 or 8.7, 8.7 or 7.6; 512: 11.3 or 10.2, 9.3 both; 640: 13.4 or 15.3, 11.0 or 12.4; 1024: 16.8 or 18.7, 15.7 or 16.4.
inline bool paged_apart(int dtype, int64_t tiles) { return tiles <= (dtype == THK_BF16 ? 4 : 2) * kCUs; }
hipError_t launch_paged_write(int dtype, int bits, const PagedWriteArgs &a, hipStream_t st);

struct PagedReadArgs {
  PagedPool p;
  void *k_out, *v_out;            // either may be nullptr
  const int32_t *n_rows, *row0;   // [B]; row0 may be nullptr (0)
  int64_t out_rows;               // rows per unit of the outputs
  int64_t most;                   // most rows of a sequence in this call
  int64_t units;
  int32_t T, ld, tiles;           // tiles: blocks per unit
  Divisor by_tiles;
  bool apart;
};
hipError_t launch_paged_read(int dtype, int bits, const PagedReadArgs &a, hipStream_t st);

struct RaggedAppendArgs {
  const void *k_new, *v_new;
  void *k_tail, *v_tail;
  const int32_t *src_row0, *n_new, *s_tail;   // [B]; src_row0 and n_new may be nullptr (0, 1)
  int64_t units;
  int32_t N_kv, B, src_rows, cap, rows;       // rows: most rows of a sequence in this call
};
hipError_t launch_append_ragged(int dtype, const RaggedAppendArgs &a, hipStream_t st);

struct PagedDecodeArgs {
  PagedPool p;
  const void *q, *kt, *vt;
  const int16_t *idx;
  const int32_t *s_pages, *s_tail;   // [B]; s_tail may be nullptr (no tail)
  void *out;
  float *ws;                         // a record per block and head of it: (max, sum, acc[128])
  int64_t S;                         // most rows of a sequence in pages
  int64_t units;
  int32_t T, G, cap, groups;         // groups: blocks of 16 query heads per unit
  int32_t n_split;                   // pieces per unit: at most, or where they go by the lengths on average
  int32_t per;                       // tiles of a piece; 0: by the lengths
  int32_t cols;                      // units and groups of one sequence: L * N_kv * groups
  int32_t step;                      // tiles a wave takes at once, at most what its kernel can
  float scale_log2;
  Divisor by_cols, by_groups, by_split;
};

// Tiles that a wave of the call's kernel can take at once.
inline int paged_decode_step(int bits, int G, int T) {
  if (bits == 4) return G <= 4 && T <= 96 ? 4 : G <= 8 ? 2 : 1;
  return bits == 8 && G <= 8 && T <= 96 ? 2 : 1;
}
hipError_t launch_paged_decode(int dtype, int bits, const PagedDecodeArgs &a, hipStream_t st);
hipError_t launch_paged_decode_bf16(int bits, const PagedDecodeArgs &a, hipStream_t st);
hipError_t launch_paged_decode_f32(int bits, const PagedDecodeArgs &a, hipStream_t st);

}  // namespace thk
