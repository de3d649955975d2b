// checks.h -- the argument checks that the entry points on logits share (host only).
#pragma once

#include <stdint.h>

#include "albireo.h"

namespace {

// Logits, shape and params (may be NULL): everything that can be told without the device.
inline albireo_status_t check_common(const void* logits, albireo_dtype_t dtype, int64_t B, int64_t V, int64_t ld,
                              const albireo_params_t* params) {
  if (dtype != ALBIREO_F32 && dtype != ALBIREO_BF16) return ALBIREO_E_INVALID;
  if (B < 0 || V <= 0 || ld < V) return ALBIREO_E_INVALID;
  if (V >= ((int64_t)1 << 31) - 16 || B >= ((int64_t)1 << 31)) return ALBIREO_E_UNSUPPORTED;
  if (B > 0 && !logits) return ALBIREO_E_INVALID;
  const int es = dtype == ALBIREO_BF16 ? 2 : 4;
  if (reinterpret_cast<uintptr_t>(logits) % es) return ALBIREO_E_INVALID;
  if (params && params->hist_offsets) {
    if (params->hist_len < 0) return ALBIREO_E_INVALID;
    if (params->hist_len > 0 && !params->hist_ids) return ALBIREO_E_INVALID;
  }
  if (params && params->prompt_offsets) {
    if (params->prompt_len < 0) return ALBIREO_E_INVALID;
    if (params->prompt_len > 0 && !params->prompt_ids) return ALBIREO_E_INVALID;
  }
  if (params && params->state) {
    const albireo_penalty_state_t* st = params->state;
    if (params->hist_offsets || params->prompt_offsets) return ALBIREO_E_INVALID;
    if (st->cap < 1 || st->cap > ALBIREO_MAX_STATE_ENTRIES) return ALBIREO_E_INVALID;
    if (B > 0 && (!st->ids || !st->counts || !st->len || !st->flags)) return ALBIREO_E_INVALID;
  }
  return ALBIREO_OK;
}

}  // namespace
