// Stand-ins for the kernel launchers of the 8-bit paged cache and of rotary positions (csrc/paged8.h) in the
// host-only sanitizer harness of their C ABI: they launch nothing and count the calls.
#include "paged8.h"

extern "C" long mf_stub_launches = 0;

namespace mf {

static hipError_t ok() { ++mf_stub_launches; return hipSuccess; }

hipError_t launch_paged8_write(const Paged8View&, const uint16_t*, int64_t, const uint16_t*, int64_t, const int32_t*, int,
                               hipStream_t) { return ok(); }
hipError_t launch_paged8_gather(const Paged8View&, const int32_t*, uint16_t*, uint16_t*, int, hipStream_t) { return ok(); }
hipError_t launch_paged8_attn(const Paged8AttnArgs&, hipStream_t) { return ok(); }
hipError_t launch_rope(const RopeArgs&, const RopePlan&, hipStream_t) { return ok(); }

}  // namespace mf
