/* The plan of a call of many query rows (csrc/tvq_rows.h), compiled for the host, for the checks in
 * test_rows_plan.py. */
#include "../../paper_2603_27467_amd/csrc/tvq_rows.h"

extern "C" void plan(int64_t batch, int64_t heads, int64_t rows, int64_t tokens, int32_t d, int64_t cus,
                     int64_t* out) {
  const tvq::RowsPlan p = tvq::rows_plan(batch, heads, rows, tokens, d, cus);
  const int64_t v[13] = {p.waves, p.unit_rows, p.tile, p.n_rb, p.n_split, p.min_tiles, p.units,
                         p.acc_bytes, p.ml_bytes, p.n_tiles, p.tile_bytes, p.exp_bytes, p.ws_bytes};
  for (int i = 0; i < 13; ++i) out[i] = v[i];
}

/* the spans of a unit, and the first tile of each and of one more; the number of spans */
extern "C" uint32_t spans(uint32_t tiles, uint32_t n_split, uint32_t min_tiles, uint32_t* start) {
  const uint32_t n = tvq::row_spans(tiles, n_split, min_tiles);
  for (uint32_t k = 0; k <= n; ++k) start[k] = tvq::span_start(tiles, n, k);
  return n;
}
