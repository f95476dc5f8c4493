// Internal view of an 8-bit cache of keys and values (sn_cache) in the kernels.
#pragma once

#include "entry_util.h"

namespace sn {

struct CacheView {
  uint8_t* k;
  uint8_t* v;
  float* k_scale;
  float* v_scale;
  int64_t pages, code_page, scale_page;  // strides of pages in elements
  int32_t heads, page, page_shift, head_dim;
};

// Checks the description and fills in its defaults.
int view_cache(const sn_cache* c, CacheView& view, bool need_memory);

}  // namespace sn
