// What the C ABI's host files share: the error text, tags, and the checks that several entry points make.
#pragma once

#include "../../include/ciar.h"

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ciar {

// Formats the calling thread's error text and returns `code`.
__attribute__((format(printf, 2, 3))) int fail(int code, const char* fmt, ...);
int hip_fail(hipError_t e, const char* what);

// The launchers report hipGetLastError() after a launch.  HIP keeps that state per host thread and a successful call
// does not reset it, so an error left by an earlier, unrelated call of the thread is discarded before the first
// launch of an entry point: what is reported afterwards is this call's.
inline void discard_stale_hip_error() { (void)hipGetLastError(); }

// Tags for the words that kernels keep in caller memory (see window_arrive in ciar_device.h): a different
// one for every launch of the process, starting from a value that varies from run to run.  (A captured graph replays
// a launch with its tag: the kernel hands every word back, with a zero tag, when a window is complete.)
uint32_t next_tag();

// The fields of ciar_params that say how logit rows lie: struct_size, vocab, dtype, window, row_stride, reserved.
int check_row_params(const ciar_params* p);

}  // namespace ciar
