// What the host files of the library share: the thread's last error. Not part
// of the C ABI.
#pragma once

#include <hip/hip_runtime.h>

#include "raas.h"

namespace raas {

// Stores the message that raas_last_error returns and gives `st` back.
raas_status fail(raas_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
raas_status hip_fail(hipError_t e, const char* what);

// Bytes of keys and values that this process's steps and attention over shared
// prefixes have read, per device: a hint that chooses between two kinds of load
// (non_temporal_loads). Adds `bytes` and gives the count before.
unsigned long long count_streamed(int device, unsigned long long bytes);
// Whether the stream is being captured into a graph.
bool capturing(hipStream_t s);

}  // namespace raas
