// Launches that do nothing, for the host side of the paged cache without a device: a handle
// can be made, and a call that is not refused says LDR_OK.
#include <hip/hip_runtime.h>

#include "serve_internal.h"

namespace ldr {
hipError_t launch_pages_reset(const PagesShape&, const PagesPtrs&, hipStream_t) { return hipSuccess; }
hipError_t launch_pages_clear_flags(const PagesPtrs&, hipStream_t) { return hipSuccess; }
hipError_t launch_pages_reserve(const PagesShape&, const PagesPtrs&, const int32_t*, int, hipStream_t) {
  return hipSuccess;
}
hipError_t launch_pages_write(const PagesShape&, const PagesPtrs&, int, int, const void*, const void*,
                              int, hipStream_t) {
  return hipSuccess;
}
hipError_t launch_pages_read(const PagesShape&, const PagesPtrs&, int, int, const int32_t*,
                             const int32_t*, void*, void*, int, hipStream_t) {
  return hipSuccess;
}
hipError_t launch_pages_keep(const PagesShape&, const PagesPtrs&, const int32_t*, hipStream_t) {
  return hipSuccess;
}
hipError_t launch_pages_fork(const PagesShape&, const PagesPtrs&, const int32_t*, hipStream_t) {
  return hipSuccess;
}
hipError_t launch_pages_compact(const PagesShape&, const PagesPtrs&, hipStream_t) { return hipSuccess; }
size_t attend_workspace_bytes(const PagesShape&, int, int) { return 256; }
hipError_t launch_attend_plan(const PagesShape&, const PagesPtrs&, int, int, const int32_t*, void*,
                              hipStream_t) {
  return hipSuccess;
}
hipError_t launch_attend(const PagesShape&, const PagesPtrs&, int, const void*, long, int, int, float,
                         void*, float*, void*, hipStream_t) {
  return hipSuccess;
}
}  // namespace ldr
