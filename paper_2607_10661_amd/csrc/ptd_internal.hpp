// Internal launchers and checks shared between translation units of the library.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ptd_common.hpp"

int ptd_launch_tree_mask(const int32_t* parent, const int32_t* tree_len, int B, int T,
                         uint64_t* mask, int32_t* depth, int32_t* dev_status,
                         hipStream_t stream);

// A page state's pointers and sizes; *shift: log2 of the page size.
static inline int ptd_check_state(const ptd_page_state* s, int* shift) {
  PTD_RETURN_IF(!s || !s->page_table || !s->num_held || !s->free_pages || !s->num_free, PTD_ERR_NULL);
  const int ps = s->page_size;
  PTD_RETURN_IF(ps < 1 || ps > (1 << 20) || (ps & (ps - 1)) != 0, PTD_ERR_SHAPE);
  PTD_RETURN_IF(s->B < 1 || s->B > 65536 || s->max_pages < 1 || s->num_pages < 1, PTD_ERR_SHAPE);
  PTD_RETURN_IF(static_cast<long long>(s->max_pages) * ps > 0x7FFFFFFFLL ||
                    static_cast<long long>(s->num_pages) * ps > 0x7FFFFFFFLL,
                PTD_ERR_SHAPE);
  int sh = 0;
  while ((1 << sh) < ps) ++sh;
  *shift = sh;
  return PTD_OK;
}
