// Instances of the paged cache's attention: one object per cache type (RR_TY)
// and width (RR_D), set by the build.
#include "rr_paged_impl.hpp"

#define RR_CAT3(a, b, c) a##b##_##c
#define RR_NAME(ty, d) RR_CAT3(launch_paged_, ty, d)

namespace rr {

hipError_t RR_NAME(RR_TY, RR_D)(const PagedArgs &a, hipStream_t stream) { return paged::launch_d<RR_TY, RR_D>(a, stream); }

}  // namespace rr
