// Per-launch timing with HIP events recorded on the launch stream. Off by
// default; when enabled every kernel launch of the library is bracketed by
// two events and attributed to a label.
#pragma once

#include <hip/hip_runtime.h>

namespace pf {

bool trace_on();
void trace_begin(const char* label, hipStream_t stream);
void trace_end(hipStream_t stream);

// f's launches under a label; the last launch error.
template <class F>
hipError_t timed(const char* label, hipStream_t s, F&& f) {
  const bool tr = trace_on();
  if (tr) trace_begin(label, s);
  f();
  const hipError_t e = hipGetLastError();
  if (tr) trace_end(s);
  return e;
}

}  // namespace pf
