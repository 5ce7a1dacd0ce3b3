// What the files of the host layer share: the calling thread's message, status
// returns, alignment checks.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "sense.h"

namespace sense {

// Keeps the message for sense_last_error_message() and returns the status
// (sense_api.hip); ok() clears it.
__attribute__((format(printf, 2, 3))) sense_status_t fail(sense_status_t st, const char* fmt, ...);
sense_status_t ok();

inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

}  // namespace sense
