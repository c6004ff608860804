// Statuses of the calls that have no model, and the checked view of a caller's cache (kv_ops.cu).
#pragma once
#include "kv_paged.h"
#include "model_view.h"

namespace adept {
// Records the message for adept_last_error(NULL) and returns s.
adept_status bad(adept_status s, const char* fmt, ...);
adept_status launched(cudaError_t e);
adept_status view_of(const adept_kv_cache* c, KvPaged* v);
}  // namespace adept
