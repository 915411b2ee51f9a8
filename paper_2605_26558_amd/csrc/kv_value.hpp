// One value of the compressed cache, for the reference read-back and for places that are visited one by one.
#pragma once
#include "cas_device.hpp"
#include "cas_internal.hpp"

namespace cas {

// bf16 word of channel col of row `row` of the tile of (layer, page, K or V, head); full == 0: the zero-padded draft view
__device__ __forceinline__ uint16_t cached_value(const KvGeom& g, const uint32_t* spec_pool, const uint32_t* verif_pool, int layer, int page, int kv,
                                                 int head, int row, int col, int full) {
  const size_t tile = (((size_t)layer * g.n_pages + page) * 2 + kv) * g.n_kv_heads + head;
  const uint32_t* ts = spec_pool + tile * g.tile_spec_words;
  const uint32_t* tv = verif_pool + tile * g.tile_verif_words;
  const uint32_t* bm = ts + row * 4;
  const int j = col >> 5, c = col & 31;
  uint32_t p = 0;
  for (int i = 0; i < j; ++i) p += __popc(bm[i]);
  const uint32_t m = bm[j];
  p += __popc(m & ((1u << c) - 1u));
  const int fw = g.mx ? 9 - g.t : 16 - g.t;
  uint32_t v;
  if ((m >> c) & 1u) {
    v = read_field(ts + g.spec_off + row * g.sw, p * fw, fw);
    const uint32_t lo = (full && g.t) ? read_field(tv + row * g.lw, p * g.t, g.t) : 0u;
    if (g.mx) {
      const int E = (int)((ts[g.page_tokens * 4 + row] >> (8 * j)) & 0xFFu);
      v = mx_word(v >> (8 - g.t), E, ((v & ((1u << (8 - g.t)) - 1u)) << g.t) | lo);
    } else {
      v = (v << g.t) | lo;
    }
  } else {
    v = full ? read_field(tv + g.page_tokens * g.lw + row * g.pw, ((uint32_t)col - p) * 16, 16) : 0u;
  }
  return (uint16_t)v;
}

}  // namespace cas
