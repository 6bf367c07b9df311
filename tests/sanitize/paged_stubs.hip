// Stand-ins for the paged cache's kernel launchers (csrc/paged.h) in the host-only sanitizer
// harness of its C ABI: they launch nothing and count the calls.
#include "paged.h"

extern "C" long mf_stub_launches = 0;

namespace mf {

static hipError_t ok() { ++mf_stub_launches; return hipSuccess; }

hipError_t launch_paged_plan(const PagedView&, const int32_t*, const int32_t*, int32_t*, int32_t*, int32_t*, int,
                             int32_t*, hipStream_t) { return ok(); }
hipError_t launch_paged_write(const PagedView&, const uint16_t*, int64_t, const uint16_t*, int64_t, const int32_t*, int,
                              hipStream_t) { return ok(); }
hipError_t launch_paged_gather(const PagedView&, const int32_t*, uint16_t*, uint16_t*, int, hipStream_t) { return ok(); }
hipError_t launch_paged_attn(const PagedAttnArgs&, hipStream_t) { return ok(); }

}  // namespace mf
