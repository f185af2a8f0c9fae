// tvq_rows.h -- attention of many query rows over the codes (tvq_rows.hip): its arguments, and how
// a call is split over workgroups.  The split is plain arithmetic, compiled into the library and,
// by itself, into the host tests.
//
// The query rows of one (sequence, KV head) are its new tokens times the G query heads, row r =
// token r / G, head r % G.  A unit is a block of consecutive rows of one (sequence, KV head) that
// a workgroup takes; the tokens that a unit attends to are cut into spans of whole tiles, one per
// workgroup, whose partials are merged.
#pragma once

#include <stdint.h>

#include "tvq_internal.h"

#if defined(__HIPCC__)
#define TVQ_ROWS_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define TVQ_ROWS_HOST_DEVICE inline
#endif

namespace tvq {

struct RowsArgs {
  Paging pg;             // pg.seq: context lengths, or tokens per (sequence, KV head) with a list
  const int32_t* list;   // [B][H][n_list] block numbers of the sequence (nullptr: all in order)
  uint32_t n_list;
  const int32_t* q_lens; // new tokens per sequence (nullptr: T)
  uint32_t B, H, G, T;   // T: token rows of q and o
  uint32_t t_end;        // bound of every context
  uint32_t cap;          // capacity tokens of a contiguous cache
  uint32_t n_rb;         // units of a (sequence, KV head)
  uint32_t n_split;      // most spans of a unit
  uint32_t min_tiles;    // fewest tiles of a span where a unit has several
  uint32_t tile;         // tokens of a tile
  uint32_t unit_rows;    // rows of a unit
  uint32_t q_f32, o_f32;
  float qscale;          // scale * log2(e): scores in log2 units
  const void* q;
  void* o;
  int64_t q_stride[3], o_stride[3];   // elements, of sequence, query head and token
  const uint32_t* signs;
  const float* lut[2];   // K and V tables: float2 entries, 1/sqrt(d) folded in
  uint32_t n[2];         // angle bins: 64, 128 or 256
  uint32_t log_norms[2]; // 4-bit log-space norms, else 8-bit linear
  const uint8_t* plane[2][3];
  float* ws_acc;         // [unit][span][unit_rows][d]
  float* ws_ml;          // [unit][span][unit_rows][2]
  uint32_t n_tiles;      // tiles of a context of t_end
  char* ws_tiles;        // rebuilt tiles [B][H][n_tiles][keys, values] (nullptr: every workgroup
  int* ws_exps;          // rebuilds its own), and their exponents
};

// Spans that a unit of `tiles` tiles is cut into.
TVQ_ROWS_HOST_DEVICE uint32_t row_spans(uint32_t tiles, uint32_t n_split, uint32_t min_tiles) {
  const uint32_t most = tiles / min_tiles;
  const uint32_t n = most < n_split ? most : n_split;
  return n < 1u ? 1u : n;
}

// First tile of span k of n.
TVQ_ROWS_HOST_DEVICE uint32_t span_start(uint32_t tiles, uint32_t n, uint32_t k) {
  const uint32_t per = tiles / n, extra = tiles - per * n;
  return k * per + (k < extra ? k : extra);
}

struct RowsPlan {
  uint32_t waves;        // of a workgroup: 4 or 8
  uint32_t unit_rows, tile, n_rb, n_split, min_tiles;
  int64_t units, acc_bytes, ml_bytes;
  int64_t n_tiles, tile_bytes, exp_bytes;   // rebuilt tiles (0: none)
  int64_t ws_bytes;
};

// Rebuilding the tiles of all tokens once costs a launch and 4 d bytes a token and head written and
// read back; every unit but one of a (sequence, KV head) is spared it.  Two sequences of 8,000 tokens,
// 8 KV heads, d = 128, us with tiles of each unit's own and kept: 2 units 70 and 77, 3 units 90 and
// 94, 4 units 107 and 106, 5 units 128 and 125, 7 units 177 and 164.  fp32 outputs would need twice
// the bytes and rebuild their own.
constexpr int64_t kRebuildUnits = 4;                 // units from which on the tiles are kept
constexpr int64_t kRebuildBytes = 1ll << 31;         // and the most they may take

// batch, heads: of the cache; rows: query rows of a (sequence, KV head); tokens: bound of a
// context; d: head dimension; cus: compute units.
//
// Up to 32 rows the four waves of a workgroup take tokens of their own, in tiles of 32 (units of 16 or
// 32 rows); above, four or eight waves of 32 rows each share tiles of 64.  Measured on both sides, us,
// 8 KV heads, d = 128:
//   4 rows, 64 blocks of 16 sequences      units of 16 rows 44, of 32 rows 55
//   20 rows, 8 sequences of 4,100 tokens   tokens of their own 38, shared tiles 45
//   32 rows, a sequence of 16,000          tokens of their own 30, shared tiles 35
//   128 rows, 8 sequences of 4,100         four waves 54, eight 59
//   256 rows, 8 sequences of 4,100         four waves (two units) 85, eight 70
// The spans of a launch go to the places that the device has for its workgroups (by their registers
// and LDS: three a compute unit with units of 16 rows, one with eight waves, else two), so many at a
// time; a span costs its tiles and, for its start and its partial, about kSpanTiles more.  The number
// of spans with the least time for full contexts is taken, of at least 4 tiles each (one a wave where
// the waves take tokens of their own).  us for several values of kSpanTiles: 448 tokens behind 7,552
// of two sequences 199 (1), 164 (3), 164 (6); with tokens of their own, one token over 512 of a
// sequence 13.2 (1), 13.2 (2), 16.7 (3) and over 256 13.2 (0), 10.9 (2), over 512 of 32 sequences 19.7
// (1), 18.7 (2), 18.7 (3).
constexpr int64_t kSpanTiles[2] = {3, 2};            // shared tiles; tokens of their own

inline RowsPlan rows_plan(int64_t batch, int64_t heads, int64_t rows, int64_t tokens, int32_t d,
                          int64_t cus) {
  const auto ceil_div = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
  RowsPlan p;
  const bool few = rows <= 32;
  p.waves = rows <= 128 ? 4 : 8;
  p.unit_rows = rows <= 16 ? 16 : few ? 32 : p.waves * 32;
  p.tile = few ? 32 : 64;
  p.min_tiles = 4;
  const int64_t n_rb = ceil_div(rows, p.unit_rows);
  p.n_rb = (uint32_t)n_rb;
  p.units = batch * heads * n_rb;
  const int64_t places = cus * (p.waves == 8 ? 1 : p.unit_rows == 16 ? 3 : 2);
  const int64_t tiles = ceil_div(tokens, p.tile);
  const int64_t fill = 4 * places / p.units + 1;      // past four rounds of places nothing is gained
  const int64_t most = tokens / (p.min_tiles * (int64_t)p.tile);
  const int64_t lanes = few ? 4 : 1;                  // waves that share a span's tiles among them
  int64_t best = 1, least = ceil_div(p.units, places) * ceil_div(tiles, lanes);
  for (int64_t n = 2; n <= most && n <= fill;) {
    const int64_t per = ceil_div(tiles, lanes * n);
    const int64_t time = ceil_div(p.units * n, places) * (per + kSpanTiles[few]);
    if (time < least) best = n, least = time;
    if (per == 1) break;
    n = ceil_div(tiles, lanes * (per - 1));           // more spans of as many tiles save nothing
  }
  p.n_split = (uint32_t)best;
  const int64_t parts = p.n_split > 1 ? p.units * p.n_split * p.unit_rows : 0;
  p.acc_bytes = (parts * d * 4 + 255) / 256 * 256;
  p.ml_bytes = (parts * 8 + 255) / 256 * 256;
  p.n_tiles = tiles;
  p.tile_bytes = batch * heads * tiles * p.tile * 4 * d;
  p.exp_bytes = batch * heads * tiles * 32;           // at most 8 groups of 4 bytes
  if (p.waves < 8 || n_rb < kRebuildUnits || p.tile_bytes > kRebuildBytes)
    p.n_tiles = p.tile_bytes = p.exp_bytes = 0;
  p.ws_bytes = p.acc_bytes + p.ml_bytes + p.tile_bytes + p.exp_bytes;
  return p;
}

}  // namespace tvq

#if defined(__HIPCC__)
int tvq_launch_rows(const tvq::RowsArgs& a, int d, unsigned waves, bool wide, void* stream);
#endif
