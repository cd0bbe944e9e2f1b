// Host helpers of the C-ABI layer, defined in abi.cpp and shared with abi_cache.cpp.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "taskpress.h"

namespace tp {

// Sets the thread's error message and returns `s`; ok() clears it and returns TP_OK.
tp_status fail(tp_status s, const char* fmt, ...);
tp_status ok();
tp_status hip_fail(hipError_t e, const char* where);
bool aligned16(const void* p);
tp_status check_dims(const tp_dims* d);
// Offsets from 0, nondecreasing (and, unless allowed, without empty entries).
tp_status check_offsets(const int64_t* off, int32_t batch, const char* what, bool allow_empty_seq);

}  // namespace tp
