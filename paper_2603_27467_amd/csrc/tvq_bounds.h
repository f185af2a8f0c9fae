// tvq_bounds.h -- arguments of the kernels that keep key bounds per pool block and choose blocks by
// them (tvq_bounds.hip), shared with the host side.
#pragma once

#include <stdint.h>

#include "tvq_internal.h"

namespace tvq {

struct KeyBoundsArgs {
  const void* k;
  int64_t stride_l;                       // elements
  uint32_t stride_b, stride_h, stride_t;  // elements, below 2^32
  uint32_t L, B, H, T;
  uint32_t n_touch;                       // blocks that T tokens of a sequence may touch
  Paging pg;                              // pg.seq: first position written
  uint16_t* bounds;                       // [L][n_blocks][H][2][d] bf16
};

struct SelectArgs {
  const uint16_t* bounds;                 // the layer's [n_blocks][H][2][d]
  const void* q;                          // [B][H*G][d]
  Paging pg;                              // pg.seq: context lengths
  uint32_t B, H, G;
  uint32_t max_ctx;
  uint32_t n_keys;                        // blocks of a context of max_ctx
  uint32_t n_sel, n_first, n_last;
  uint32_t* keys;                         // [B*H][n_keys]
  int32_t* blocks;                        // [B*H][n_sel]
  int32_t* lens;                          // [B*H]
  uint32_t cus;            // compute units
};

}  // namespace tvq

int tvq_launch_key_bounds(const tvq::KeyBoundsArgs& a, int d, bool f32, void* stream);
int tvq_launch_select(const tvq::SelectArgs& a, int d, bool f32, void* stream);
