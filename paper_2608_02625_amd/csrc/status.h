// Error reporting shared by the files that hold C entry points (engine.hip,
// cache.hip).  Not part of the library's interface.
#pragma once

#include <hip/hip_runtime.h>

#include <string>

#include "../../include/dlm.h"

// Sets the thread's message and returns s.
dlm_status dlm_internal_fail(dlm_status s, const std::string& msg);
// The status of the exception being handled; the message is set without throwing.
dlm_status dlm_internal_caught() noexcept;
// Shape, buffers and alignment of a caller's cache.
dlm_status dlm_internal_check_cache(const dlm_cache* cache);
// Sizes of windows of up to `rows` rows whose heads a call takes; "" if it may.
std::string dlm_internal_check_windows(const dlm_cache& cache, int n_heads, int64_t rows);
