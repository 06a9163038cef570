// Checks that the entry points of the 16-bit blocks share.
#pragma once
#include "rc_common.hpp"

namespace rc {

// A KV descriptor whose tokens are addressed by slots, block * T + place.
inline rc_status check_paged(const rc_kv_desc* d, int64_t n_blocks, const char* who) {
  const bool many = d && n_blocks > 0x7fffffffLL / (d->block_tokens == 32 ? 32 : 16);
  if (rc_status e = check_desc(d, many ? 0 : n_blocks, who)) return e;
  if (many) return fail(RC_ERR_UNSUPPORTED, "%s: more than 2^31 - 1 slots (n_blocks * T)", who);
  if (d->n_layers > 65535) return fail(RC_ERR_UNSUPPORTED, "%s: more than 65535 layers", who);
  return RC_OK;
}

}  // namespace rc
