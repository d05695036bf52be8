// cache8.h -- the checks of a cache in 8 bits that its operators share.
#pragma once

#include "../../include/predecoder_ops.h"
#include "token_values.h"

namespace pd {

// Sizes and type, or with the arrays.
inline pd_status check_cache(const pd_cache& c, bool arrays) {
  if (c.batch < 0 || c.kv_heads < 0 || c.capacity < 0 || c.head_dim < 1) return PD_ERR_INVALID_ARG;
  if (c.codes_type != PD_CODES_E4M3 && c.codes_type != PD_CODES_INT8) return PD_ERR_INVALID_ARG;
  if (c.head_dim % 16 || c.head_dim > 128 || c.batch > 65535 || c.kv_heads > 65535) return PD_ERR_UNSUPPORTED;
  if (!arrays) return PD_OK;
  if (!c.codes || !c.scales || !c.sites) return PD_ERR_INVALID_ARG;
  if ((uintptr_t)c.codes % 16 || (uintptr_t)c.scales % 4 || (uintptr_t)c.sites % 16) return PD_ERR_INVALID_ARG;
  return PD_OK;
}

}  // namespace pd
